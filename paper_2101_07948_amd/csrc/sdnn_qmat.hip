// Products of 4-bit weights with the activations of few tokens.
#include <type_traits>

#include "sdnn_decode_device.h"
#include "sdnn_decode_shape.h"
#include "sdnn_device.h"

namespace sdnn {
namespace {

// Layout of the weights: tiles of 16 rows, of these chunks of 128 columns, of these 16 bytes for
// each of 64 lanes.  Lane l has row l & 15; its dword j holds columns 32 j + 8 (l / 16) + i of the
// chunk, i = 0 ... 7: what the lane gives to matrix instruction j as its operand.  Column i < 4 is in the lower half of
// byte i, column 4 + i in the upper half: after a mask a byte n is the 8-bit float n 2^-9 (4 bits of exponent, 3 of
// mantissa: 0 ... 7 are its subnormals, 8 ... 15 have the least exponent).  A wave reads 1 KiB in one access.  The scales
// and zero points follow: [tile][group][16 rows] where groups are whole chunks, else [tile][chunk][16 rows][group of
// the chunk], so that a lane has those of a chunk in one access (see metas_of).
__host__ __device__ constexpr int bit_of(int i) { return i < 4 ? 8 * i : 8 * (i - 4) + 4; }
constexpr int kMaxWaves = 16;

__global__ __launch_bounds__(256) void qmat_pack(const uint8_t* packed, int32_t M, int32_t K, int32_t chunks,
                                                 int64_t first, int64_t dwords, uint32_t* out) {
  const int64_t at = first + (int64_t)blockIdx.x * 256 + threadIdx.x;  // [tile][chunk][lane][j]
  if (at >= dwords) return;
  const int j = at & 3, lane = (at >> 2) & 63;
  const int64_t tc = at >> 8;
  const int64_t row = tc / chunks * kQTileRows + (lane & 15);
  const int k0 = (int)(tc % chunks) * kQChunk + j * 32 + (lane >> 4) * 8;
  uint32_t w = 0;
  if (row < M && k0 < K) {
    const uint8_t* from = packed + row * ((K + 1) / 2) + k0 / 2;
    uint32_t eight = 0;  // numbers, 4 bits each
    if (k0 + 8 <= K)
      __builtin_memcpy(&eight, from, 4);
    else
      for (int i = 0; 2 * i < K - k0; ++i) eight |= (uint32_t)from[i] << (8 * i);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      w |= (k0 + i < K ? eight >> (4 * i) & 15u : 0) << bit_of(i);
    }
  }
  out[at] = w;
}

// Scales (of `bytes` each) and zero points in that order, zeros past M and past the last group.  `outer`: groups of
// whole chunks, or chunks; `inner`: groups of a chunk, or 1.
__global__ __launch_bounds__(256) void qmat_pack_meta(const uint8_t* scales, int32_t bytes, const uint8_t* zeros,
                                                      int32_t M, int32_t groups, int32_t outer, int32_t inner,
                                                      int64_t first, int64_t count, uint8_t* out) {
  const int64_t at = first + (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= count) return;
  const int64_t to = at / (kQTileRows * inner);
  const int64_t row = to / outer * kQTileRows + at / inner % kQTileRows;
  const int64_t group = to % outer * inner + at % inner;
  const bool there = row < M && group < groups;
  const int64_t from = row * groups + group;
  for (int i = 0; i < bytes; ++i) out[at * bytes + i] = there ? scales[from * bytes + i] : 0;
  if (zeros) out[count * bytes + at] = there ? zeros[from] : 0;
}

struct QmatArgs {
  const i32x4* weights;
  const uint8_t* scales;
  const uint8_t* zeros;  // NULL: 8
  const void* x;
  void* y;
  int64_t x_feature, x_column, y_feature, y_column;
  const float* bias;
  int32_t M, K, N, chunks;
  int32_t metas;      // groups of whole chunks of a tile, or its chunks
  uint32_t group_of;  // of chunk c, where groups are whole chunks: the upper 32 bits of c * group_of (0: c)
  int32_t scale_dtype, epi;
};

// The matrix instruction of a type.  `weights`: the 8 numbers of a dword, from the 8-bit floats that they are.
template <typename T, typename V8>
struct Op16 {
  typedef V8 type;
  template <bool UPPER>
  static __device__ __forceinline__ int32_t pair(uint32_t four) {
    if constexpr (__is_same(T, _Float16))
      return __builtin_bit_cast(int32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(four, 512.0f, UPPER));
    else
      return __builtin_bit_cast(int32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(four, 512.0f, UPPER));
  }
  static __device__ __forceinline__ V8 weights(uint32_t w) {
    const uint32_t lower = w & 0x0f0f0f0fu, upper = w >> 4 & 0x0f0f0f0fu;
    return __builtin_bit_cast(V8, i32x4{pair<false>(lower), pair<true>(lower), pair<false>(upper), pair<true>(upper)});
  }
};
template <typename T>
struct Op;
template <>
struct Op<_Float16> : Op16<_Float16, f16x8> {
  static __device__ __forceinline__ f32x4 mfma(f16x8 a, f16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
};
template <>
struct Op<__bf16> : Op16<__bf16, bf16x8> {
  static __device__ __forceinline__ f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
};
template <>
struct Op<float> : Op<__bf16> {};

// Columns of x on their way to LDS: a chunk's 128 values of up to TOKENS columns, TOKENS pairs of values to a lane.
// Where a column's values are contiguous, pair t is values 2 lane, 2 lane + 1 of column t, one load whatever its
// alignment (the hardware takes any); else (FEATURES) a lane has column lane % TOKENS, and a wave's loads are
// neighbouring columns of a few values.  Columns past the last repeat it (without conditions the loads are under way
// together).  Columns of 16 bits are a row of LDS each; 32-bit values are the exact sum of three bf16 numbers
// of 8 bits each, and have three.
constexpr int kRowBytes = kQChunk * 2 + 16;  // (16 more: the rows of one piece lie in different banks)
template <typename T, int TOKENS, bool FEATURES>
struct Columns {
  typedef T Pair __attribute__((ext_vector_type(2)));
  static constexpr int kSide = FEATURES ? 64 / TOKENS : 64;  // pairs of a column that a wave's load takes
  // As loaded: taken apart or put together only when they are stored (anything else would wait for them).
  typedef typename std::conditional<sizeof(T) == 2, uint16_t, uint32_t>::type Bits;
  Pair pair[FEATURES ? 1 : TOKENS];
  uint32_t lo[FEATURES ? TOKENS : 1], hi[FEATURES ? TOKENS : 1];
  // x: the first of the N columns, k0: the chunk's first value.  PART: K may end within.
  template <bool PART>
  __device__ __forceinline__ void load(const QmatArgs& a, const T* x, int N, int k0, int lane) {
    if constexpr (FEATURES) {
      const T* c = x + min(lane % TOKENS, N - 1) * a.x_column;
#pragma unroll
      for (int j = 0; j < TOKENS; ++j) {
        const int k = k0 + 2 * (lane / TOKENS + kSide * j);
        const int64_t u = PART ? min(k, a.K - 1) : k, v = PART ? min(k + 1, a.K - 1) : k + 1;
        lo[j] = __builtin_bit_cast(Bits, c[u * a.x_feature]), hi[j] = __builtin_bit_cast(Bits, c[v * a.x_feature]);
        if (PART) lo[j] = k < a.K ? lo[j] : 0, hi[j] = k + 1 < a.K ? hi[j] : 0;
      }
    } else {
      const int k = k0 + 2 * lane;
#pragma unroll
      for (int t = 0; t < TOKENS; ++t) {
        const T* c = x + min(t, N - 1) * a.x_column;
        if (PART) {
          const T u = c[min(k, a.K - 1)], v = c[min(k + 1, a.K - 1)];
          pair[t] = Pair{k < a.K ? u : (T)0.0f, k + 1 < a.K ? v : (T)0.0f};
        } else {
          __builtin_memcpy(&pair[t], c + k, sizeof(Pair));
        }
      }
    }
  }
  // Row t of LDS is column t; of 32-bit values rows 4 t + part with up to four columns, else TOKENS part + t.
  __device__ __forceinline__ void store(unsigned char* rows, int lane) const {
#pragma unroll
    for (int j = 0; j < TOKENS; ++j) {
      const int t = FEATURES ? lane % TOKENS : j;
      unsigned char* at = rows + (FEATURES ? lane / TOKENS + kSide * j : lane) * 4;
      if constexpr (sizeof(T) == 2) {
        if constexpr (FEATURES)
          *reinterpret_cast<uint32_t*>(at + t * kRowBytes) = lo[j] | hi[j] << 16;
        else
          *reinterpret_cast<Pair*>(at + t * kRowBytes) = pair[j];
      } else {
        float u, v;
        if constexpr (FEATURES)
          u = __uint_as_float(lo[j]), v = __uint_as_float(hi[j]);
        else
          u = pair[j][0], v = pair[j][1];
#pragma unroll
        for (int part = 0; part < 3; ++part) {  // the upper 16 bits of a float are its first 8 bits as a bf16
          const uint32_t ub = __float_as_uint(u), vb = __float_as_uint(v);
          *reinterpret_cast<uint32_t*>(at + (TOKENS <= 4 ? 4 * t + part : TOKENS * part + t) * kRowBytes) =
              __builtin_amdgcn_perm(vb, ub, 0x07060302u);
          u -= __uint_as_float(ub & 0xffff0000u), v -= __uint_as_float(vb & 0xffff0000u);
        }
      }
    }
  }
};
template <typename T, int TOKENS>
constexpr int kRowsOf = sizeof(T) == 2 ? TOKENS : TOKENS <= 4 ? 4 * TOKENS : 3 * TOKENS;

// The most waves of a workgroup; half where the registers of 16 waves do not hold the columns on their way.
template <int TOKENS, bool FEATURES>
constexpr int kWavesOf = TOKENS == 16 && FEATURES ? kMaxWaves / 2 : kMaxWaves;

// N scales from scale i on (N bytes or more apart: one access), and zero points.
template <int N>
__device__ __forceinline__ void load_scales(const QmatArgs& a, int64_t i, float (&scale)[N], float (&zero)[N]) {
  if (a.scale_dtype == SDNN_F32) {
    load_n<N>(reinterpret_cast<const float*>(a.scales) + i, true, scale);
  } else if (a.scale_dtype == SDNN_F16) {
    _Float16 s[N];
    load_n<N>(reinterpret_cast<const _Float16*>(a.scales) + i, true, s);
#pragma unroll
    for (int k = 0; k < N; ++k) scale[k] = (float)s[k];
  } else {
    __bf16 s[N];
    load_n<N>(reinterpret_cast<const __bf16*>(a.scales) + i, true, s);
#pragma unroll
    for (int k = 0; k < N; ++k) scale[k] = (float)s[k];
  }
  uint8_t z[N];
#pragma unroll
  for (int k = 0; k < N; ++k) z[k] = 8;
  if (a.zeros) load_n<N>(a.zeros + i, true, z);
#pragma unroll
  for (int k = 0; k < N; ++k) zero[k] = (float)z[k];
}

// A chunk of a tile on its way to the registers: 16 bytes of weights, scales and zeros, and the columns of x.
template <typename T, int STEPS, int TOKENS, bool FEATURES>
struct Chunk {
  i32x4 w;
  float scale[4 / STEPS], zero[4 / STEPS];
  Columns<T, TOKENS, FEATURES> x;
  // w0: of the lane in the first chunk; meta0: the lane's row of the first scales.
  template <bool PART>
  __device__ __forceinline__ void load(const QmatArgs& a, const i32x4* w0, const T* x0, int N, int64_t meta0, int c,
                                       int lane) {
    w = w0[(int64_t)c * 64];
    const int meta = STEPS == 4 && a.group_of ? (int)__umulhi((uint32_t)c, a.group_of) : c;
    load_scales<4 / STEPS>(a, meta0 + (int64_t)meta * (kQTileRows * (4 / STEPS)), scale, zero);
    x.template load<PART>(a, x0, N, c * kQChunk, lane);
    __builtin_amdgcn_sched_barrier(0);  // under way before the chunk before is multiplied
  }
};

// A workgroup has 16 rows of W and up to TOKENS columns of x; its waves share the chunks, each with the next one
// under way while it multiplies.  The columns go through LDS (a wave's own part), where they are turned into
// operands: rows of the first operand are columns of x, columns of the second rows of W.  With n the 4-bit numbers,
// a group adds s (sum n x - z sum x): both sums come from the matrix unit, the second with ones for the numbers, and are
// scaled once a group (and chunk).  (With 16 + n and 16 + z in their place the sums were 2.5 times as inexact.)
//   Row p of the operand is column p / 4 + 4 (p % 4) of x, so that up to four columns are in the first of a lane's
// four results, up to eight in two; of four columns in 32 bits rows 4 t + part, and a lane adds its results.
//   Reading the weights bounds it: 16384 x 8192 with one column in 16 bits 14.1 us, 69 MB at 4.9 TB/s, the rate of a
// large copy.  5003 x 4099 with 13 columns: 11.5 us for 12.5 MB: each of 313 workgroups, one or two to a compute unit,
// brings all of x through LDS.  Small ones are a launch: 768 x 3072 3.8 us.
//   STEPS: matrix instructions (of 32 columns of W) of a group within a chunk.
template <typename T, int STEPS, int TOKENS, bool FEATURES>
__global__ __launch_bounds__((kWavesOf<TOKENS, FEATURES> * 64)) void qmat_kernel(QmatArgs a) {
  constexpr bool PARTS = sizeof(T) == 4, PACKED = PARTS && TOKENS <= 4;
  constexpr int REGS = TOKENS < 4 ? 1 : TOKENS / 4, SETS = PARTS && !PACKED ? 3 : 1, ROWS = kRowsOf<T, TOKENS>;
  extern __shared__ __align__(16) unsigned char lds[];  // a wave's rows, then its sums
  const int lane = threadIdx.x % 64, r = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), waves = blockDim.x / 64;
  const int64_t tile = blockIdx.x;
  const int n0 = blockIdx.y * TOKENS, N = min(TOKENS, a.N - n0);
  const T* x = static_cast<const T*>(a.x) + n0 * a.x_column;
  const i32x4* w = a.weights + tile * a.chunks * 64 + lane;
  const int64_t meta0 = (tile * a.metas * kQTileRows + r) * (4 / STEPS);
  unsigned char* rows = lds + wave * ROWS * kRowBytes;
  const unsigned char* row =
      rows + (PACKED ? 4 * min(r >> 2, TOKENS - 1) + min(r & 3, 2) : min((r >> 2) + 4 * (r & 3), TOKENS - 1)) * kRowBytes +
      g * 16;  // (rows of the operand that are no column repeat one)
  float acc[REGS] = {};
  typename Op<T>::type ones;
#pragma unroll
  for (int i = 0; i < 8; ++i) ones[i] = 1.0f;
  const auto add = [&](const Chunk<T, STEPS, TOKENS, FEATURES>& b) {
    b.x.store(rows, lane);
    // what the lanes of the wave wrote, before they read each other's
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
    for (int i = 0; i < 4 / STEPS; ++i) {
      f32x4 d = {0, 0, 0, 0}, sx = {0, 0, 0, 0};
      // Two lower parts of 32-bit values first: added to the sums of the upper ones they would round to these, 3 times a
      // step (5 to 8 columns: 2.8 times the error).
#pragma unroll
      for (int pass = SETS > 1; pass >= 0; --pass) {
#pragma unroll
        for (int s = i * STEPS; s < (i + 1) * STEPS; ++s) {
          uint32_t bits = (uint32_t)b.w[s];
          if (SETS > 1) asm volatile("" : "+v"(bits));  // (made again in each pass: kept, the numbers would cost a wave)
          const auto wv = Op<T>::weights(bits);
#pragma unroll
          for (int k = pass ? SETS - 1 : 0; k >= pass; --k) {
            const auto xv = *reinterpret_cast<const typename Op<T>::type*>(row + s * 64 + k * TOKENS * kRowBytes);
            d = Op<T>::mfma(xv, wv, d);
            sx = Op<T>::mfma(xv, ones, sx);
          }
        }
      }
      const float s = b.scale[i], z = b.zero[i];
      if (PACKED) {
        acc[0] = fmaf(s, fmaf(-z, (sx[0] + sx[1]) + sx[2], (d[0] + d[1]) + d[2]), acc[0]);
      } else {
#pragma unroll
        for (int k = 0; k < REGS; ++k) acc[k] = fmaf(s, fmaf(-z, sx[k], d[k]), acc[k]);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
  };
  const int whole = a.K / kQChunk;  // chunks; of one more, K ends within
  {
    Chunk<T, STEPS, TOKENS, FEATURES> even, odd;
    int c = wave;
    if (c < whole) even.template load<false>(a, w, x, N, meta0, c, lane);
    for (; c < whole; c += 2 * waves) {
      if (c + waves < whole) odd.template load<false>(a, w, x, N, meta0, c + waves, lane);
      add(even);
      if (c + waves >= whole) break;
      if (c + 2 * waves < whole) even.template load<false>(a, w, x, N, meta0, c + 2 * waves, lane);
      add(odd);
    }
  }
  if (whole < a.chunks && wave == whole % waves) {
    Chunk<T, STEPS, TOKENS, FEATURES> last;
    last.template load<true>(a, w, x, N, meta0, whole, lane);
    add(last);
  }
  __syncthreads();
  float* sums = reinterpret_cast<float*>(lds);  // [wave][REGS][64]
#pragma unroll
  for (int i = 0; i < REGS; ++i) sums[(wave * REGS + i) * 64 + lane] = acc[i];
  __syncthreads();
  if (wave >= REGS) return;
  float v = 0.0f;
  for (int k = 0; k < waves; ++k) v += sums[(k * REGS + wave) * 64 + lane];
  const int64_t m = tile * kQTileRows + r;
  const int n = n0 + g + 4 * wave;  // row 4 g + wave of the result
  if (m >= a.M || n >= a.N) return;
  v += a.bias ? a.bias[m] : 0.0f;
  static_cast<T*>(a.y)[m * a.y_feature + n * a.y_column] = (T)activation(v, a.epi);
}

template <typename T, int STEPS, int TOKENS>
hipError_t start_tokens(const QmatArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)((a.M + kQTileRows - 1) / kQTileRows), (unsigned)((a.N + TOKENS - 1) / TOKENS));
  // 8 waves to a tile of rows, 16 where there are fewer tiles than compute units (1000 x 12000, 4 columns in 32 bits:
  // 12.0 and 9.7 us; 227 x 11127, 16 contiguous columns in 16 bits: 11.3 and 10.5), with as many chunks each as the one with most
  // of them; 4 at least, which write the results
  constexpr size_t per_wave = (size_t)kRowsOf<T, TOKENS> * kRowBytes;
  const int most = grid.x * grid.y >= 256 ? 8 : a.x_feature == 1 ? kWavesOf<TOKENS, false> : kWavesOf<TOKENS, true>;
  const int each = (a.chunks + most - 1) / most, needed = (a.chunks + each - 1) / each;
  const int waves = needed < 4 ? 4 : needed;
  constexpr size_t sums = (TOKENS < 4 ? 4 : TOKENS) * 64;  // of a wave
  const size_t lds = waves * (per_wave > sums ? per_wave : sums);
  const auto kernel = a.x_feature == 1 ? qmat_kernel<T, STEPS, TOKENS, false> : qmat_kernel<T, STEPS, TOKENS, true>;
  if (lds > 65536) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  kernel<<<grid, waves * 64, lds, stream>>>(a);
  return hipGetLastError();
}

template <typename T, int STEPS>
hipError_t start_steps(const QmatArgs& a, hipStream_t stream) {
  if (a.N == 1) return start_tokens<T, STEPS, 1>(a, stream);
  if (a.N <= 4) return start_tokens<T, STEPS, 4>(a, stream);
  if constexpr (sizeof(T) == 2)
    if (a.N > 8) return start_tokens<T, STEPS, 16>(a, stream);
  return start_tokens<T, STEPS, 8>(a, stream);  // (the three parts of 16 in 32 bits do not fit the registers)
}

template <typename T>
hipError_t start(const QmatArgs& a, int group, hipStream_t stream) {
  if (group == 32) return start_steps<T, 1>(a, stream);
  if (group == 64) return start_steps<T, 2>(a, stream);
  return start_steps<T, 4>(a, stream);
}

}  // namespace

hipError_t launch_qmat_pack(const sdnn_qmat_s& w, const uint8_t* packed, const void* scales,
                            const uint8_t* zeros, hipStream_t stream) {
  const int64_t dwords = qmat_weight_bytes(w) / 4, entries = scales_of(w);
  constexpr int64_t most = (int64_t)1 << 31;  // threads of a launch
  for (int64_t first = 0; first < dwords; first += most)
    qmat_pack<<<(unsigned)((std::min(dwords - first, most) + 255) / 256), 256, 0, stream>>>(
        packed, w.M, w.K, w.chunks, first, dwords, reinterpret_cast<uint32_t*>(const_cast<uint8_t*>(w.weights)));
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  for (int64_t first = 0; first < entries; first += most)
    qmat_pack_meta<<<(unsigned)((std::min(entries - first, most) + 255) / 256), 256, 0, stream>>>(
        static_cast<const uint8_t*>(scales), dtype_bytes(w.scale_dtype), zeros, w.M, groups_of(w), metas_of(w), inner_of(w),
        first, entries, const_cast<uint8_t*>(w.meta));
  return hipGetLastError();
}

hipError_t launch_qmat(const sdnn_qmat_s& w, const void* x, int64_t x_feature, int64_t x_column, void* y,
                       int64_t y_feature, int64_t y_column, int32_t N, int dtype, const float* bias,
                       int epi, hipStream_t stream) {
  QmatArgs a = {};
  a.weights = reinterpret_cast<const i32x4*>(w.weights);
  a.scales = w.meta;
  a.metas = metas_of(w);
  a.zeros = w.zeros ? w.meta + scales_of(w) * dtype_bytes(w.scale_dtype) : nullptr;
  a.x = x, a.x_feature = x_feature, a.x_column = x_column;
  a.y = y, a.y_feature = y_feature, a.y_column = y_column;
  if (w.K == 1) a.x_feature = 1;  // one value is contiguous
  a.bias = bias, a.M = w.M, a.K = w.K, a.N = N, a.chunks = w.chunks;
  const uint32_t group_chunks = w.group / kQChunk;  // (c < 2^13, group_chunks < 2^24: the quotients are exact)
  a.group_of = group_chunks > 1 ? (uint32_t)(((1ull << 32) + group_chunks - 1) / group_chunks) : 0;
  a.scale_dtype = w.scale_dtype, a.epi = epi;
  if (dtype == SDNN_F32) return start<float>(a, w.group, stream);
  if (dtype == SDNN_F16) return start<_Float16>(a, w.group, stream);
  return start<__bf16>(a, w.group, stream);
}

}  // namespace sdnn
