// The choice of the next token.
#include "sdnn_decode_device.h"
#include "sdnn_serve_shape.h"

// Every operation is rounded by itself, so that a token's weight is the same wherever it is computed.
#pragma clang fp contract(off)

namespace sdnn {
namespace {

constexpr int kThreads = kSampleThreads, kWavesOf = kThreads / 64;
constexpr int kBins = kSampleBins, kPerThread = kBins / kThreads;
constexpr int kOctaves = 46;  // a weight below 2^-kUnit is none
constexpr int kUnit = 44;     // weights are whole numbers of 2^-kUnit
constexpr int kList = 2048;   // tokens that are put in order in LDS

struct SampleArgs {
  const void* logits;
  int64_t row_stride;
  int32_t vocab;
  const float* u;
  sdnn_sampling settings;
  int32_t* token;
  float* logprob;
};

// What a row's weights are made by.
struct Weights {
  float top;     // the largest logit
  double scale;  // log2 e / temperature
};

// The exponent of a token's weight, not above 0.  (Where the largest logit is infinite, its like have 0 and all others -infinity.)
__device__ __forceinline__ double exponent_of(const Weights& w, float l) {
  return l == w.top ? 0.0 : l == -INFINITY ? -INFINITY : ((double)l - (double)w.top) * w.scale;
}
// 2^z as a whole number of 2^-kUnit: the fraction's power is a float of 24 bits, shifted by the whole part.
__device__ __forceinline__ uint64_t weight_of(double z) {
  if (!(z > -(double)kOctaves)) return 0;
  const double n = rint(z);
  const float x = __builtin_amdgcn_exp2f((float)(z - n)) * 0x1p23f;
  return ((uint64_t)(uint32_t)x << (kUnit - 23)) >> -(int)n;
}
__device__ __forceinline__ int bin_of(double z) {
  constexpr double PER = (double)kBins / kOctaves;
  return z > -(double)kOctaves ? min((int)(-z * PER), kBins - 1) : kBins - 1;
}

// Tokens in order: larger logits first, equal ones by index.  (-0 and 0 are equal.)
__device__ __forceinline__ uint64_t order_of(float l, int i) {
  const int32_t b = __float_as_int(l == 0.0f ? 0.0f : l);
  const uint32_t ascending = (uint32_t)b ^ (b < 0 ? 0xffffffffu : 0x80000000u);
  return (uint64_t)~ascending << 32 | (uint32_t)i;
}
__device__ __forceinline__ float logit_of(uint64_t order) {
  const uint32_t ascending = ~(uint32_t)(order >> 32);
  return __uint_as_float(ascending & 0x80000000u ? ascending ^ 0x80000000u : ~ascending);
}

// A row, read in pieces of 16 bytes that lie where 16-byte loads may; those at its ends value by value.  Piece g has the
// tokens g V - lead ... g V - lead + V - 1.
template <typename T>
struct Row {
  static constexpr int V = 16 / sizeof(T);
  const T* x;
  int lead, pieces, vocab;
  __device__ __forceinline__ Row(const SampleArgs& a, int r) {
    x = static_cast<const T*>(a.logits) + r * a.row_stride;
    vocab = a.vocab;
    lead = (int)((uintptr_t)x % 16 / sizeof(T));
    pieces = (lead + vocab + V - 1) / V;
  }
  // The tokens' logits, NaN as -infinity; -infinity also past the row's ends.
  __device__ __forceinline__ void load(int g, float (&l)[V]) const {
    const int i = g * V - lead;
    T v[V];
    if (i >= 0 && i + V <= vocab) {
      load_n<V>(x + i, true, v);
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) v[e] = i + e >= 0 && i + e < vocab ? x[i + e] : (T)-INFINITY;
    }
#pragma unroll
    for (int e = 0; e < V; ++e) {
      l[e] = (float)v[e];
      l[e] = l[e] == l[e] ? l[e] : -INFINITY;
    }
  }
  // f(index, logit) of all tokens of pieces begin, begin + step ... below end, several loads under way at once.
  template <typename F>
  __device__ __forceinline__ void each(int begin, int end, int step, const F& f) const {
    constexpr int AHEAD = 4;
    for (int g = begin; g < end; g += AHEAD * step) {
      float l[AHEAD][V];
#pragma unroll
      for (int k = 0; k < AHEAD; ++k)
        if (g + k * step < end) load(g + k * step, l[k]);
#pragma unroll
      for (int k = 0; k < AHEAD; ++k)
        if (g + k * step < end) {
#pragma unroll
          for (int e = 0; e < V; ++e) f((g + k * step) * V - lead + e, l[k][e]);
        }
    }
  }
};

struct SampleLds {
  uint64_t mass[kBins];
  uint32_t count[kBins];
  uint64_t list[kList];
  uint64_t masses[kWavesOf];
  uint32_t counts[kWavesOf];
  float tops[kWavesOf];
  // what one thread finds for all
  uint64_t found_mass;
  uint32_t found_count;
  int32_t found, listed;
  uint64_t found_order;
};

__device__ __forceinline__ uint64_t wave_sum(uint64_t x) {
#pragma unroll
  for (int s = 32; s; s >>= 1) x += __shfl_xor((unsigned long long)x, s);
  return x;
}

// Which of `n` consecutive entries, kPerThread (at most) to a thread, is the one with which the running sums, counts or
// masses, pass `target` (0 <= target < the sum of all); left in l.found with the sums before it.
template <int PER>
__device__ __forceinline__ void find_entry(SampleLds& l, const uint32_t* count, const uint64_t* mass, bool by_count, uint64_t target) {
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  uint64_t m = 0;
  uint32_t c = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) m += mass[threadIdx.x * PER + i], c += count[threadIdx.x * PER + i];
  uint64_t m1 = m;
  uint32_t c1 = c;
#pragma unroll
  for (int s = 1; s < 64; s *= 2) {
    const uint64_t y = __shfl_up((unsigned long long)m1, s);
    const uint32_t z = __shfl_up(c1, s);
    if (lane >= s) m1 += y, c1 += z;
  }
  if (lane == 63) l.masses[wave] = m1, l.counts[wave] = c1;
  __syncthreads();
  uint64_t m0 = m1 - m;
  uint32_t c0 = c1 - c;
  for (int w = 0; w < wave; ++w) m0 += l.masses[w], c0 += l.counts[w];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const uint64_t me = mass[threadIdx.x * PER + i];
    const uint32_t ce = count[threadIdx.x * PER + i];
    const uint64_t before = by_count ? c0 : m0, with = before + (by_count ? ce : me);
    if (before <= target && target < with) l.found = threadIdx.x * PER + i, l.found_mass = m0, l.found_count = c0;
    m0 += me, c0 += ce;
  }
  __syncthreads();
}

// The last token that is kept of bin `bin`: the one with which the running sums of the bin's tokens in their order, counts
// or masses, pass `target`; left in l.found_order, with the mass before it in the bin in l.found_mass.
template <typename T>
__device__ void resolve(SampleLds& l, const Row<T>& row, const Weights& w, int bin, uint32_t tokens, bool by_count, uint64_t target) {
  const int tid = threadIdx.x;
  if (tokens <= kList) {
    if (tid == 0) l.listed = 0;
    __syncthreads();
    row.each(tid, row.pieces, kThreads, [&](int i, float x) {
      if (x > -INFINITY && bin_of(exponent_of(w, x)) == bin) {
        const int at = atomicAdd(&l.listed, 1);
        if (at < kList) l.list[at] = order_of(x, i);
      }
    });
    int n = 64;
    while (n < (int)tokens) n *= 2;
    __syncthreads();
    for (int i = l.listed + tid; i < n; i += kThreads) l.list[i] = ~0ull;
    __syncthreads();
    for (int size = 2; size <= n; size *= 2)
      for (int step = size / 2; step; step /= 2) {
        for (int i = tid; i < n / 2; i += kThreads) {
          const int a = (i & ~(step - 1)) * 2 + (i & (step - 1)), b = a + step;
          const uint64_t x = l.list[a], y = l.list[b];
          if ((x > y) == ((a & size) == 0)) l.list[a] = y, l.list[b] = x;
        }
        __syncthreads();
      }
    // running sums, kList / kThreads tokens to a thread
    constexpr int PER = kList / kThreads;
    const int lane = tid % 64, wave = tid / 64;
    uint64_t m[PER], sum = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int at = tid * PER + i;
      m[i] = at < (int)tokens ? weight_of(exponent_of(w, logit_of(l.list[at]))) : 0;
      sum += m[i];
    }
    uint64_t m1 = sum;
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
      const uint64_t y = __shfl_up((unsigned long long)m1, s);
      if (lane >= s) m1 += y;
    }
    if (lane == 63) l.masses[wave] = m1;
    __syncthreads();
    uint64_t m0 = m1 - sum;
    for (int v = 0; v < wave; ++v) m0 += l.masses[v];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int at = tid * PER + i;
      const uint64_t before = by_count ? at : m0, with = before + (by_count ? 1 : m[i]);
      if (at < (int)tokens && before <= target && target < with) l.found_order = l.list[at], l.found_mass = m0;
      m0 += m[i];
    }
    __syncthreads();
    return;
  }
  // More tokens than the list holds: digit by digit, 8 bits of the 64 of a token's place in the order.
  uint64_t prefix = 0, mass_before = 0;
  for (int digit = 56; digit >= 0; digit -= 8) {
    for (int i = tid; i < kThreads; i += kThreads) l.mass[i] = 0, l.count[i] = 0;
    __syncthreads();
    row.each(tid, row.pieces, kThreads, [&](int i, float x) {
      if (!(x > -INFINITY)) return;
      const double z = exponent_of(w, x);
      const uint64_t v = order_of(x, i);
      if (bin_of(z) != bin || (digit < 56 && v >> (digit + 8) != prefix >> (digit + 8))) return;
      const int d = (int)(v >> digit & 255);
      atomicAdd(&l.count[d], 1u);
      atomicAdd(reinterpret_cast<unsigned long long*>(&l.mass[d]), (unsigned long long)weight_of(z));
    });
    __syncthreads();
    find_entry<1>(l, l.count, l.mass, by_count, target);
    prefix |= (uint64_t)l.found << digit;
    target -= by_count ? l.found_count : l.found_mass;
    mass_before += l.found_mass;
    __syncthreads();
  }
  if (tid == 0) l.found_order = prefix, l.found_mass = mass_before;
  __syncthreads();
}

// A row to a workgroup.  Of the passes over it (the largest logit; the bins' counts and masses; the tokens of the bins that the
// limits fall into; the masses kept) those that a row's settings do not ask for are left out; all but the first read from L2.
template <typename T>
__global__ __launch_bounds__(kThreads) void sample_kernel(SampleArgs a) {
  extern __shared__ __align__(16) unsigned char raw[];
  SampleLds& l = *reinterpret_cast<SampleLds*>(raw);
  const int r = blockIdx.x, tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  const Row<T> row(a, r);
  const sdnn_sampling& s = a.settings;
  const float temperature = s.temperature ? s.temperature[r] : 1.0f;
  const bool greedy = !(temperature > 0.0f);
  const int top_k = s.top_k && s.top_k[r] > 0 && s.top_k[r] < a.vocab ? s.top_k[r] : 0;
  const float top_p = s.top_p && s.top_p[r] < 1.0f ? s.top_p[r] : 1.0f;
  const float min_p = s.min_p && s.min_p[r] > 0.0f ? s.min_p[r] : 0.0f;

  // the largest logit, and the first token that has it
  float top = -INFINITY;
  int at = 0x7fffffff;
  row.each(tid, row.pieces, kThreads, [&](int i, float x) {
    if (x > top) top = x, at = i;
  });
  uint64_t first = order_of(top, at);  // (a thread's first: its tokens ascend)
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    const uint64_t y = __shfl_xor((unsigned long long)first, d);
    first = y < first ? y : first;
  }
  if (lane == 0) l.masses[wave] = first;
  __syncthreads();
  for (int v = 0; v < kWavesOf; ++v) first = l.masses[v] < first ? l.masses[v] : first;
  __syncthreads();
  const Weights w = {logit_of(first), 1.4426950408889634 / (double)temperature};
  if (w.top == -INFINITY || greedy || top_k == 1 || !(top_p > 0.0f) || min_p > 1.0f) {
    if (tid == 0) {
      a.token[r] = w.top == -INFINITY ? -1 : (int32_t)(uint32_t)first;
      if (a.logprob) a.logprob[r] = w.top == -INFINITY ? -INFINITY : 0.0f;
    }
    return;
  }

  uint64_t last = ~0ull;  // of the tokens that are kept, in their order
  if (top_k > 0 || top_p < 1.0f) {
    const auto fill_bins = [&] {
      for (int i = tid; i < kBins; i += kThreads) l.mass[i] = 0, l.count[i] = 0;
      __syncthreads();
      uint64_t all = 0;
      row.each(tid, row.pieces, kThreads, [&](int, float x) {
        if (!(x > -INFINITY)) return;
        const double z = exponent_of(w, x);
        const uint64_t m = weight_of(z);
        const int b = bin_of(z);
        all += m;
        atomicAdd(&l.count[b], 1u);
        atomicAdd(reinterpret_cast<unsigned long long*>(&l.mass[b]), (unsigned long long)m);
      });
      all = wave_sum(all);
      if (lane == 0) l.masses[wave] = all;
      __syncthreads();
      all = 0;
      for (int v = 0; v < kWavesOf; ++v) all += l.masses[v];
      __syncthreads();
      return all;
    };
    uint64_t kept = fill_bins();
    if (top_k > 0) {
      if (tid == 0) l.found = -1;
      __syncthreads();
      find_entry<kPerThread>(l, l.count, l.mass, true, (uint64_t)(top_k - 1));
      const int bin = l.found;  // -1: fewer tokens than that have a logit; those in the last bin have no weight
      if (bin >= 0 && bin < kBins - 1) {
        const uint64_t before = l.found_mass;
        const uint32_t tokens = l.count[bin], rank = (uint32_t)(top_k - 1) - l.found_count;
        __syncthreads();
        resolve(l, row, w, bin, tokens, true, rank);
        last = l.found_order;
        kept = before + l.found_mass + weight_of(exponent_of(w, logit_of(last)));
        __syncthreads();
        if (tokens > kList && top_p < 1.0f) fill_bins();  // (whose place was taken)
      }
    }
    const double limit = (double)top_p * (double)kept;
    if (top_p < 1.0f) {
      // the last token whose weights before it sum to less than the limit: the one with which they reach it
      const uint64_t target = (uint64_t)ceil(limit) - 1;
      if (target < kept) {
        find_entry<kPerThread>(l, l.count, l.mass, false, target);
        const int b = l.found;
        const uint64_t rest = target - l.found_mass;
        const uint32_t tokens = l.count[b];
        __syncthreads();
        resolve(l, row, w, b, tokens, false, rest);
        last = l.found_order < last ? l.found_order : last;
        __syncthreads();
      }
    }
  }

  // The masses kept, by index: of 16 parts of the row, then of 16 parts of the one that the token lies in, until a wave has
  // few enough pieces to look at them one by one.
  const double least = min_p > 0.0f ? log2((double)min_p) : -INFINITY;
  const auto kept_weight = [&](int i, float x) -> uint64_t {
    if (!(x > -INFINITY) || order_of(x, i) > last) return 0;
    const double z = exponent_of(w, x);
    return z >= least ? weight_of(z) : 0;
  };
  int begin = 0, end = row.pieces;
  uint64_t before = 0, total = 0, target = 0;
  bool whole = true;
  for (;;) {
    const int part = (end - begin + kWavesOf - 1) / kWavesOf;
    const int from = min(begin + wave * part, end), to = min(from + part, end);
    uint64_t m = 0;
    row.each(from + lane, to, 64, [&](int i, float x) { m += kept_weight(i, x); });
    m = wave_sum(m);
    if (lane == 0) l.masses[wave] = m;
    __syncthreads();
    if (whole) {
      for (int v = 0; v < kWavesOf; ++v) total += l.masses[v];
      const float u = a.u[r];
      const double x = (double)(u > 0.0f ? u : 0.0f) * (double)total;
      target = x < (double)total ? (uint64_t)x : total;
      if (target >= total) target = total - 1;
      whole = false;
    }
    int v = 0;
    while (v < kWavesOf - 1 && before + l.masses[v] <= target) before += l.masses[v], ++v;
    __syncthreads();
    begin = min(begin + v * part, end), end = min(begin + part, end);
    if (part <= 64) break;
  }
  if (wave > 0) return;
  // a piece to a lane
  constexpr int V = Row<T>::V;
  float x[V];
  uint64_t m[V], sum = 0;
  const int g = begin + lane;
  if (g < end) row.load(g, x);
#pragma unroll
  for (int e = 0; e < V; ++e) {
    m[e] = g < end ? kept_weight(g * V - row.lead + e, x[e]) : 0;
    sum += m[e];
  }
  uint64_t run = sum;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint64_t y = __shfl_up((unsigned long long)run, d);
    if (lane >= d) run += y;
  }
  run += before - sum;
#pragma unroll
  for (int e = 0; e < V; ++e) {
    if (run <= target && target < run + m[e]) {
      a.token[r] = g * V - row.lead + e;
      if (a.logprob)
        a.logprob[r] = (float)((exponent_of(w, x[e]) + ((double)kUnit - log2((double)total))) * 0.6931471805599453);
    }
    run += m[e];
  }
}

template <typename T>
hipError_t start(const SampleArgs& a, int32_t rows, hipStream_t stream) {
  const auto kernel = sample_kernel<T>;
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize,
                                           (int)sizeof(SampleLds));
  if (e != hipSuccess) return e;
  kernel<<<(unsigned)rows, kThreads, sizeof(SampleLds), stream>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_sample(const void* logits, int64_t row_stride, int dtype, int32_t rows, int32_t vocab, const float* u,
                         const sdnn_sampling& settings, int32_t* token, float* logprob, float*, hipStream_t stream) {
  if (!launchable(rows, kThreads)) return hipErrorInvalidConfiguration;
  SampleArgs a = {};
  a.logits = logits, a.row_stride = row_stride, a.vocab = vocab, a.u = u, a.settings = settings;
  a.token = token, a.logprob = logprob;
  return dtype == SDNN_F32   ? start<float>(a, rows, stream)
         : dtype == SDNN_F16 ? start<_Float16>(a, rows, stream)
                             : start<__bf16>(a, rows, stream);
}

}  // namespace sdnn
