// The choice of blocks by the score of their summaries.
#include "sdnn_decode_device.h"

namespace sdnn {
namespace {

struct SelectArgs {
  const void* q;
  int64_t q_token, q_head;
  const int8_t* means;
  const float* scales;
  int64_t pages;
  const int32_t* pos;
  const int32_t* seq;
  const int32_t* table;
  int32_t* chosen;
  int32_t tokens, sequences, max_blocks;
  int32_t kv_heads, group, head_dim, block_shift;
  int32_t blocks, sink, local;
};

// A number whose order as an unsigned integer is the order of the floats (-0 counts as 0).
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  return u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
}

// 16 bytes of a summary from byte k on, zeros past its end (D is a multiple of 8).
__device__ __forceinline__ i32x4 load_mean(const int8_t* row, int k, int D, bool wide) {
  i32x4 v = {0, 0, 0, 0};
  if (wide) {
    if (k < D) v = *reinterpret_cast<const i32x4*>(row + k);
  } else {
    if (k < D) {
      const int2 lo = *reinterpret_cast<const int2*>(row + k);
      v[0] = lo.x, v[1] = lo.y;
    }
    if (k + 8 < D) {
      const int2 hi = *reinterpret_cast<const int2*>(row + k + 8);
      v[2] = hi.x, v[3] = hi.y;
    }
  }
  return v;
}

// Sums of two counts over the workgroup's threads before this one.  `parts`: a word for each wave.
__device__ __forceinline__ uint2 before(uint2 n, uint2* parts) {
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  uint2 s = n;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t x = __shfl_up(s.x, d), y = __shfl_up(s.y, d);
    if (lane >= d) s.x += x, s.y += y;
  }
  __syncthreads();
  if (lane == 63) parts[wave] = s;
  __syncthreads();
  uint2 r = make_uint2(s.x - n.x, s.y - n.y);
  for (int w = 0; w < wave; ++w) r.x += parts[w].x, r.y += parts[w].y;
  return r;
}

// A workgroup chooses the blocks of one token and cached head.  The dot products of 16 summaries
// with up to 16 queries are one matrix instruction for 64 values of a head: bytes in, whole
// numbers out.  The scores go to LDS as ordered integers; the value of the last one taken is found
// by counting them by their bytes from the top, four times, and a scan over the blocks in order
// writes out what is above it and as many equal to it as are still wanted.
template <typename T, int STEPS>
__global__ __launch_bounds__(1024) void select_kernel(SelectArgs a) {
  extern __shared__ __align__(16) unsigned char lds[];
  const int group16 = (a.group + 15) & ~15;
  int8_t* m8 = reinterpret_cast<int8_t*>(lds);                        // [group16][STEPS * 64]
  float* top = reinterpret_cast<float*>(m8 + group16 * STEPS * 64);   // [group16]
  uint32_t* bins = reinterpret_cast<uint32_t*>(top + group16);        // [256]
  uint2* parts = reinterpret_cast<uint2*>(bins + 256);                // [16]
  uint32_t* found = reinterpret_cast<uint32_t*>(parts + 16);          // [2]
  uint32_t* key = found + 2;                                          // [max_blocks]
  const int threads = blockDim.x, lane = threadIdx.x % 64, wave = threadIdx.x / 64, waves = threads / 64;
  const int h = blockIdx.x % a.kv_heads, t = blockIdx.x / a.kv_heads;
  int32_t* chosen = a.chosen + ((int64_t)t * a.kv_heads + h) * a.blocks;
  const int32_t p = a.pos[t], seq = a.seq[t];
  const int n = p < 0 || (uint32_t)seq >= (uint32_t)a.sequences ? 0 : min((p >> a.block_shift) + 1, a.max_blocks);
  if (n <= a.blocks) {  // everything the token sees
    for (int i = threadIdx.x; i < a.blocks; i += threads) chosen[i] = i < n ? i : -1;
    return;
  }
  for (int i = threadIdx.x; i < a.sink; i += threads) chosen[i] = i;
  for (int i = threadIdx.x; i < a.local; i += threads) chosen[a.blocks - a.local + i] = n - a.local + i;
  const int count = n - a.sink - a.local;             // blocks to choose from, from block `sink` on
  const uint32_t take = a.blocks - a.sink - a.local;  // of them; less than count
  if (take == 0) return;
  const int D = a.head_dim, row_bytes = STEPS * 64;
  for (int g = wave; g < group16; g += waves) {
    const T* q = static_cast<const T*>(a.q) + t * a.q_token + (int64_t)(h * a.group + g) * a.q_head;
    float x[STEPS], m = 0.0f;
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const int d = s * 64 + lane;
      x[s] = g < a.group && d < D ? (float)q[d] : 0.0f;
      m = fmaxf(m, fabsf(x[s]));
    }
#pragma unroll
    for (int s = 32; s; s >>= 1) m = fmaxf(m, __shfl_xor(m, s));
    const float f = m > 0.0f ? 127.0f * (1.0f / m) : 0.0f;
#pragma unroll
    for (int s = 0; s < STEPS; ++s)
      m8[g * row_bytes + s * 64 + lane] = (int8_t)fminf(fmaxf(rintf(x[s] * f), -127.0f), 127.0f);
    if (lane == 0) top[g] = m;
  }
  __syncthreads();

  const int32_t* table = a.table + (int64_t)seq * a.max_blocks + a.sink;
  const int r = lane & 15, kg = lane >> 4;
  const bool wide = D % 16 == 0;
  for (int b0 = wave * 16; b0 < count; b0 += waves * 16) {
    int64_t page = b0 + r < count ? table[b0 + r] : -1;
    if (page >= a.pages) page = -1;
    const int64_t row = max(page, (int64_t)0) * a.kv_heads + h;
    i32x4 m[STEPS];
#pragma unroll
    for (int s = 0; s < STEPS; ++s) m[s] = load_mean(a.means + row * D, s * 64 + kg * 16, D, wide);
    const float scale = a.scales[row];
    float best[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    for (int g0 = 0; g0 < group16; g0 += 16) {
      i32x4 dot = {0, 0, 0, 0};
#pragma unroll
      for (int s = 0; s < STEPS; ++s) {
        const i32x4 qv = *reinterpret_cast<const i32x4*>(m8 + (g0 + r) * row_bytes + s * 64 + kg * 16);
        dot = __builtin_amdgcn_mfma_i32_16x16x64_i8(m[s], qv, dot, 0, 0, 0);
      }
      const float tq = top[g0 + r];
#pragma unroll
      for (int i = 0; i < 4; ++i)  // row kg * 4 + i of the 16 blocks, query g0 + r
        if (g0 + r < a.group) best[i] = fmaxf(best[i], (float)dot[i] * tq);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int s = 8; s; s >>= 1) best[i] = fmaxf(best[i], __shfl_xor(best[i], s));
      // the scale and the page of block kg * 4 + i are in lane kg * 4 + i
      const float sb = __shfl(scale, kg * 4 + i);
      const int64_t pg = __shfl(page, kg * 4 + i);
      const int b = b0 + kg * 4 + i;
      if (r == 0 && b < count) key[b] = pg < 0 ? 0u : ordered(best[i] * sb);
    }
  }

  uint32_t prefix = 0, want = take;  // `want` of the keys that begin with prefix are taken
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = threadIdx.x; i < 256; i += threads) bins[i] = 0;
    __syncthreads();
    const uint32_t mask = shift == 24 ? 0u : 0xffffffffu << (shift + 8);
    for (int i = threadIdx.x; i < count; i += threads) {
      const uint32_t k = key[i];
      if ((k & mask) == prefix) atomicAdd(&bins[(k >> shift) & 255], 1u);
    }
    __syncthreads();
    if (wave == 0) {  // lane l has bins 255 - 4 l - 3 ... 255 - 4 l, counted from the top
      uint32_t c[4], sum = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) c[i] = bins[255 - 4 * lane - i], sum += c[i];
      uint32_t above = sum;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const uint32_t x = __shfl_up(above, d);
        if (lane >= d) above += x;
      }
      above -= sum;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (above < want && want <= above + c[i]) {
          found[0] = prefix | (uint32_t)(255 - 4 * lane - i) << shift;
          found[1] = want - above;
        }
        above += c[i];
      }
    }
    __syncthreads();
    prefix = found[0], want = found[1];
  }

  const int run = (count + threads - 1) / threads;  // blocks of a thread, in order
  const int i0 = min((int)threadIdx.x * run, count), i1 = min(i0 + run, count);
  uint2 mine = make_uint2(0, 0);
  for (int i = i0; i < i1; ++i) {
    const uint32_t k = key[i];
    mine.x += k > prefix, mine.y += k == prefix;
  }
  const uint2 b = before(mine, parts);
  uint32_t equal = b.y, at = a.sink + b.x + min(b.y, want);
  for (int i = i0; i < i1; ++i) {
    const uint32_t k = key[i];
    if (k > prefix || (k == prefix && equal++ < want)) chosen[at++] = a.sink + i;
  }
}

template <typename T, int STEPS>
hipError_t start(const SelectArgs& a, unsigned grid, int threads, size_t lds, hipStream_t stream) {
  if (lds > 65536) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(select_kernel<T, STEPS>),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  select_kernel<T, STEPS><<<grid, threads, lds, stream>>>(a);
  return hipGetLastError();
}

template <typename T>
hipError_t start_steps(const SelectArgs& a, unsigned grid, int threads, size_t lds, hipStream_t stream) {
  if (a.head_dim <= 64) return start<T, 1>(a, grid, threads, lds, stream);
  if (a.head_dim <= 128) return start<T, 2>(a, grid, threads, lds, stream);
  return start<T, 4>(a, grid, threads, lds, stream);
}

}  // namespace

hipError_t launch_select(const sdnn_block_cache& c, const sdnn_tokens& t, const sdnn_heads& q,
                         int32_t blocks, int32_t sink, int32_t local, int32_t* chosen, hipStream_t stream) {
  SelectArgs a = {};
  a.q = q.data, a.q_token = q.token_stride, a.q_head = q.head_stride;
  a.means = c.means, a.scales = c.mean_scales, a.pages = c.pages;
  a.pos = t.pos, a.seq = t.seq, a.table = t.table, a.chosen = chosen;
  a.tokens = t.tokens, a.sequences = t.sequences, a.max_blocks = t.max_blocks;
  a.kv_heads = c.kv_heads, a.group = q.heads / c.kv_heads, a.head_dim = c.head_dim;
  a.block_shift = __builtin_ctz(c.block);
  a.blocks = blocks, a.sink = sink, a.local = local;
  const int steps = c.head_dim <= 64 ? 1 : c.head_dim <= 128 ? 2 : 4;
  const int group16 = (a.group + 15) & ~15;
  const size_t lds = (size_t)group16 * (steps * 64 + 4) + 256 * 4 + 16 * 8 + 8 + (size_t)t.max_blocks * 4;
  const unsigned grid = (unsigned)t.tokens * c.kv_heads;
  const int threads = t.max_blocks > 1024 ? 1024 : t.max_blocks > 256 ? 256 : 64;
  if (c.dtype == SDNN_F32) return start_steps<float>(a, grid, threads, lds, stream);
  if (c.dtype == SDNN_F16) return start_steps<_Float16>(a, grid, threads, lds, stream);
  return start_steps<__bf16>(a, grid, threads, lds, stream);
}

}  // namespace sdnn
