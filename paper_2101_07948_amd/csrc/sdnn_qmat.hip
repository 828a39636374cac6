// Products of 4-bit weights with the activations of few tokens.
#include "sdnn_decode_device.h"
#include "sdnn_device.h"

namespace sdnn {
namespace {

// Layout of the weights: tiles of 16 rows, of these chunks of 128 columns, of these 16 bytes for
// each of 64 lanes.  Lane l has row l & 15; its dword j holds columns 32 j + 8 (l / 16) + i of the
// chunk, i = 0 ... 7, number i at bit 8 i (i < 4) or 8 (i - 4) + 4: what the lane gives to matrix
// instruction j as its operand, one mask and four byte conversions for each half.  A wave reads
// 1 KiB in one access.  The scales and zero points follow: [tile][group][16 rows].
constexpr int kMaxWaves = 16;

__global__ __launch_bounds__(256) void qmat_pack(const uint8_t* packed, int32_t M, int32_t K, int32_t chunks,
                                                 int64_t dwords, uint32_t* out) {
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;  // [tile][chunk][lane][j]
  if (at >= dwords) return;
  const int j = at & 3, lane = (at >> 2) & 63;
  const int64_t tc = at >> 8;
  const int64_t row = tc / chunks * kQTileRows + (lane & 15);
  const int k0 = (int)(tc % chunks) * kQChunk + j * 32 + (lane >> 4) * 8;
  uint32_t w = 0;
  if (row < M)
    for (int i = 0; i < 8; ++i) {
      const int k = k0 + i;
      if (k >= K) break;
      const uint32_t b = packed[row * ((K + 1) / 2) + k / 2];
      w |= (k & 1 ? b >> 4 : b & 15) << (i < 4 ? 8 * i : 8 * (i - 4) + 4);
    }
  out[at] = w;
}

// scales (of `bytes` each) and zero points to [tile][group][16 rows]; rows past M get zeros.
__global__ __launch_bounds__(256) void qmat_pack_meta(const uint8_t* scales, int32_t bytes, const uint8_t* zeros,
                                                      int32_t M, int32_t groups, int64_t count, uint8_t* out) {
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= count) return;
  const int64_t tg = at / kQTileRows;
  const int64_t row = tg / groups * kQTileRows + at % kQTileRows;
  const int64_t from = row * groups + tg % groups;
  for (int i = 0; i < bytes; ++i) out[at * bytes + i] = row < M ? scales[from * bytes + i] : 0;
  if (zeros) out[count * bytes + at] = row < M ? zeros[from] : 0;
}

struct QmatArgs {
  const i32x4* weights;
  const uint8_t* scales;
  const uint8_t* zeros;  // NULL: 8
  const void* x;
  void* y;
  int64_t x_feature, x_column, y_feature, y_column;
  const float* bias;
  int32_t M, K, N, chunks, groups, group_chunks;  // chunks of a group of 128 columns or more
  int32_t scale_dtype, epi;
};

// What a lane gives to the matrix instruction of columns [k, k + 8) for the column of x that it has: the values
// as loaded, and as the operand.
template <typename T>
struct Operand;

// 8 values from x + k * x_feature on.  Contiguous ones come in 16-byte loads whatever their alignment (the
// hardware takes any; one by one, the 13 columns of an odd-sized layer took 7 times as long).
template <typename T>
__device__ __forceinline__ void load8(const T* x, const QmatArgs& a, int k, T (&v)[8]) {
  if (k + 8 <= a.K) {
    if (a.x_feature == 1) {
      __builtin_memcpy(v, x + k, sizeof(v));
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = x[(k + i) * a.x_feature];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = k + i < a.K ? x[(k + i) * a.x_feature] : (T)0.0f;
  }
}

template <typename T, typename V8>
struct Operand16 {
  typedef V8 type;
  static constexpr int kTokens = 16;
  // Row p of the operand is column p / 4 + 4 (p % 4) of x: with up to four columns, the results are in
  // the first of a lane's four registers.
  static __device__ __forceinline__ int token(int p) { return (p >> 2) + 4 * (p & 3); }
  static __device__ __forceinline__ V8 operand(const T (&v)[8], int) { return *reinterpret_cast<const V8*>(v); }
  static __device__ __forceinline__ V8 weights(uint32_t w) {
    const uint32_t lo = w & 0x0f0f0f0fu, hi = (w >> 4) & 0x0f0f0f0fu;
    V8 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[i] = (T)(float)((lo >> (8 * i)) & 255u);
      v[4 + i] = (T)(float)((hi >> (8 * i)) & 255u);
    }
    return v;
  }
};
template <>
struct Operand<_Float16> : Operand16<_Float16, f16x8> {
  static __device__ __forceinline__ f32x4 mfma(f16x8 a, f16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
};
template <>
struct Operand<__bf16> : Operand16<__bf16, bf16x8> {
  static __device__ __forceinline__ f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
};
// 32-bit activations as the exact sum of three bf16 numbers of 8 bits each, in three rows of the
// operand: row p is part p % 4 of column p / 4 (part 3: nothing).  The 4-bit numbers are exact in
// bf16, so every product is exact.
template <>
struct Operand<float> {
  typedef bf16x8 type;
  static constexpr int kTokens = 4;
  static __device__ __forceinline__ int token(int p) { return p >> 2; }
  static __device__ __forceinline__ bf16x8 operand(const float (&f)[8], int part) {
    const float second = part >= 1 ? 1.0f : 0.0f, third = part >= 2 ? 1.0f : 0.0f;
    bf16x8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) {  // the upper 16 bits of a float are its first 8 bits as a bf16
      float r = f[i];
      r -= second * __uint_as_float(__float_as_uint(r) & 0xffff0000u);
      r -= third * __uint_as_float(__float_as_uint(r) & 0xffff0000u);
      v[i] = __builtin_bit_cast(__bf16, (uint16_t)(__float_as_uint(r) >> 16));
    }
    return v;
  }
  static __device__ __forceinline__ bf16x8 weights(uint32_t w) { return Operand<__bf16>::weights(w); }
  static __device__ __forceinline__ f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) { return Operand<__bf16>::mfma(a, b, c); }
};

__device__ __forceinline__ float scale_at(const QmatArgs& a, int64_t i) {
  if (a.scale_dtype == SDNN_F32) return reinterpret_cast<const float*>(a.scales)[i];
  if (a.scale_dtype == SDNN_F16) return (float)reinterpret_cast<const _Float16*>(a.scales)[i];
  return (float)reinterpret_cast<const __bf16*>(a.scales)[i];
}

// A chunk of a tile on its way to the registers: 16 bytes of weights, the lane's column of x, scales and zeros.
template <typename T, int STEPS>
struct Chunk {
  i32x4 w;
  T x[4][8];
  float scale[4 / STEPS], zero[4 / STEPS];
  __device__ __forceinline__ void load(const QmatArgs& a, const i32x4* w0, const T* x0, bool live, int64_t meta0,
                                       int c, int g) {
    w = w0[(int64_t)c * 64];
#pragma unroll
    for (int i = 0; i < 4 / STEPS; ++i) {
      // (a group past the last, where K ends within the chunk, meets zeros of x)
      const int group = STEPS == 4 ? c / a.group_chunks : min(c * (4 / STEPS) + i, a.groups - 1);
      const int64_t at = meta0 + (int64_t)group * kQTileRows;
      scale[i] = scale_at(a, at);
      zero[i] = a.zeros ? (float)a.zeros[at] : 8.0f;
    }
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      if (live) {
        load8(x0, a, c * kQChunk + s * 32 + g * 8, x[s]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[s][i] = (T)0.0f;
      }
    }
    __builtin_amdgcn_sched_barrier(0);  // under way before the chunk before is multiplied
  }
};

// A workgroup has 16 rows of W and up to 16 columns of x (4 in 32 bits); its waves share the chunks, each with
// the next one under way while it multiplies.  With n the 4-bit numbers, a group of columns adds
// s (sum n x - z sum x): both sums come from the matrix unit, the second with ones for the numbers, and are
// scaled once a group.  What bounds it: reading the weights (half a byte each; the conversion takes two vector
// instructions of 64 lanes for 64 of them).
//   STEPS: matrix instructions (of 32 columns) of a group within a chunk.
//   REGS: of a lane's four result registers, those that hold columns of x.
template <typename T, int STEPS, int REGS>
__global__ __launch_bounds__(kMaxWaves * 64) void qmat_kernel(QmatArgs a) {
  typedef Operand<T> Op;
  constexpr bool kParts = sizeof(T) == 4;
  __shared__ float sums[kMaxWaves][REGS][64];
  const int lane = threadIdx.x % 64, r = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), waves = blockDim.x / 64;
  const int64_t tile = blockIdx.x;
  const int n0 = blockIdx.y * Op::kTokens, part = r & 3;
  const int token = n0 + Op::token(r);
  const bool live = token < a.N && !(kParts && part == 3);
  const T* x = static_cast<const T*>(a.x) + (live ? token : 0) * a.x_column;
  const i32x4* w = a.weights + tile * a.chunks * 64 + lane;
  const int64_t meta0 = tile * a.groups * kQTileRows + r;
  float acc[REGS] = {};
  typename Op::type ones;
#pragma unroll
  for (int i = 0; i < 8; ++i) ones[i] = 1.0f;
  const auto add = [&](const Chunk<T, STEPS>& b) {
#pragma unroll
    for (int i = 0; i < 4 / STEPS; ++i) {
      f32x4 d = {0, 0, 0, 0}, sx = {0, 0, 0, 0};
#pragma unroll
      for (int s = i * STEPS; s < (i + 1) * STEPS; ++s) {
        const auto xv = Op::operand(b.x[s], part);
        d = Op::mfma(xv, Op::weights((uint32_t)b.w[s]), d);
        sx = Op::mfma(xv, ones, sx);
      }
      const float s = b.scale[i], z = b.zero[i];
      if (kParts) {
        acc[0] = fmaf(s, fmaf(-z, (sx[0] + sx[1]) + sx[2], (d[0] + d[1]) + d[2]), acc[0]);
      } else {
#pragma unroll
        for (int k = 0; k < REGS; ++k) acc[k] = fmaf(s, fmaf(-z, sx[k], d[k]), acc[k]);
      }
    }
  };
  Chunk<T, STEPS> even, odd;
  int c = wave;
  if (c < a.chunks) even.load(a, w, x, live, meta0, c, g);
  for (; c < a.chunks; c += 2 * waves) {
    if (c + waves < a.chunks) odd.load(a, w, x, live, meta0, c + waves, g);
    add(even);
    if (c + waves >= a.chunks) break;
    if (c + 2 * waves < a.chunks) even.load(a, w, x, live, meta0, c + 2 * waves, g);
    add(odd);
  }
#pragma unroll
  for (int i = 0; i < REGS; ++i) sums[wave][i][lane] = acc[i];
  __syncthreads();
  if (wave >= REGS) return;
  float v = 0.0f;
  for (int k = 0; k < waves; ++k) v += sums[k][wave][lane];
  const int64_t m = tile * kQTileRows + r;
  const int n = n0 + g + 4 * wave;  // row 4 g + wave of the result
  if (m >= a.M || n >= a.N) return;
  v += a.bias ? a.bias[m] : 0.0f;
  static_cast<T*>(a.y)[m * a.y_feature + n * a.y_column] = (T)activation(v, a.epi);
}

template <typename T, int STEPS>
hipError_t start_regs(const QmatArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)((a.M + kQTileRows - 1) / kQTileRows),
                  (unsigned)((a.N + Operand<T>::kTokens - 1) / Operand<T>::kTokens));
  // 8 waves to a tile of rows, 16 where there are fewer tiles than compute units; not more than chunks
  const int most = grid.x * grid.y < 256 ? kMaxWaves : 8;
  int waves = 4;
  while (waves < most && waves < a.chunks) waves *= 2;
  if (sizeof(T) == 4 || a.N <= 4)
    qmat_kernel<T, STEPS, 1><<<grid, waves * 64, 0, stream>>>(a);
  else if (a.N <= 8)
    qmat_kernel<T, STEPS, sizeof(T) == 4 ? 1 : 2><<<grid, waves * 64, 0, stream>>>(a);
  else
    qmat_kernel<T, STEPS, sizeof(T) == 4 ? 1 : 4><<<grid, waves * 64, 0, stream>>>(a);
  return hipGetLastError();
}

template <typename T>
hipError_t start(const QmatArgs& a, int group, hipStream_t stream) {
  if (group == 32) return start_regs<T, 1>(a, stream);
  if (group == 64) return start_regs<T, 2>(a, stream);
  return start_regs<T, 4>(a, stream);
}

int64_t groups_of(const sdnn_qmat_s& w) { return (w.K + w.group - 1) / w.group; }

}  // namespace

int64_t qmat_weight_bytes(const sdnn_qmat_s& w) { return (int64_t)w.tiles * w.chunks * 1024; }
int64_t qmat_meta_bytes(const sdnn_qmat_s& w) {
  return w.tiles * groups_of(w) * kQTileRows * (dtype_bytes(w.scale_dtype) + (w.zeros ? 1 : 0));
}

hipError_t launch_qmat_pack(const sdnn_qmat_s& w, const uint8_t* packed, const void* scales,
                            const uint8_t* zeros, hipStream_t stream) {
  const int64_t dwords = qmat_weight_bytes(w) / 4, entries = w.tiles * groups_of(w) * kQTileRows;
  qmat_pack<<<(unsigned)((dwords + 255) / 256), 256, 0, stream>>>(
      packed, w.M, w.K, w.chunks, dwords, reinterpret_cast<uint32_t*>(const_cast<uint8_t*>(w.weights)));
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  qmat_pack_meta<<<(unsigned)((entries + 255) / 256), 256, 0, stream>>>(
      static_cast<const uint8_t*>(scales), dtype_bytes(w.scale_dtype), zeros, w.M, (int32_t)groups_of(w), entries,
      const_cast<uint8_t*>(w.meta));
  return hipGetLastError();
}

hipError_t launch_qmat(const sdnn_qmat_s& w, const void* x, int64_t x_feature, int64_t x_column, void* y,
                       int64_t y_feature, int64_t y_column, int32_t N, int dtype, const float* bias,
                       int epi, hipStream_t stream) {
  QmatArgs a = {};
  a.weights = reinterpret_cast<const i32x4*>(w.weights);
  a.scales = w.meta;
  a.groups = (int32_t)groups_of(w);
  a.zeros = w.zeros ? w.meta + (int64_t)w.tiles * a.groups * kQTileRows * dtype_bytes(w.scale_dtype) : nullptr;
  a.x = x, a.x_feature = x_feature, a.x_column = x_column;
  a.y = y, a.y_feature = y_feature, a.y_column = y_column;
  a.bias = bias, a.M = w.M, a.K = w.K, a.N = N, a.chunks = w.chunks;
  a.group_chunks = w.group >= kQChunk ? w.group / kQChunk : 1;
  a.scale_dtype = w.scale_dtype, a.epi = epi;
  if (dtype == SDNN_F32) return start<float>(a, w.group, stream);
  if (dtype == SDNN_F16) return start<_Float16>(a, w.group, stream);
  return start<__bf16>(a, w.group, stream);
}

}  // namespace sdnn
