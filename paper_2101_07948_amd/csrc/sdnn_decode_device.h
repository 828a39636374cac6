// Device code shared by the kernels of sdnn_decode.h: element types, vector loads of rows of
// any alignment, and the rotation.
#ifndef SDNN_DECODE_DEVICE_H_
#define SDNN_DECODE_DEVICE_H_

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sdnn_decode_internal.h"

namespace sdnn {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

template <int N, typename T>
struct VecOf {
  typedef T type __attribute__((ext_vector_type(N)));
};
template <typename T>
struct VecOf<1, T> {
  typedef T type;
};

// N consecutive values at p: one load or store where `aligned` (p a multiple of the vector's
// size), else N.  `aligned` is uniform over a launch.
template <int N, typename T>
__device__ __forceinline__ void load_n(const T* p, bool aligned, T (&out)[N]) {
  if (aligned) {
    const auto v = *reinterpret_cast<const typename VecOf<N, T>::type*>(p);
    __builtin_memcpy(out, &v, sizeof(out));
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) out[i] = p[i];
  }
}
template <int N, typename T>
__device__ __forceinline__ void store_n(T* p, bool aligned, const T (&in)[N]) {
  if (aligned) {
    typename VecOf<N, T>::type v;
    __builtin_memcpy(&v, in, sizeof(in));
    *reinterpret_cast<typename VecOf<N, T>::type*>(p) = v;
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = in[i];
  }
}

// 16 bytes from global memory to LDS, one piece a lane: lane l's goes to `to` + 16 l (`to` is uniform over
// the wave).
__device__ __forceinline__ void copy_to_lds(const void* from, unsigned char* to) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from,
                                   (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}

// x and the value of the lane 16 (32) away, exchanged within the registers (gfx950's row swaps: with the same
// value as both operands, one result holds the even rows twice and the other the odd ones).
__device__ __forceinline__ void with_16(float x, float* u, float* v) {
  const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  *u = __uint_as_float(p[0]), *v = __uint_as_float(p[1]);
}
__device__ __forceinline__ void with_32(float x, float* u, float* v) {
  const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  *u = __uint_as_float(p[0]), *v = __uint_as_float(p[1]);
}
__device__ __forceinline__ float max_over_16(float x) {
  float u, v;
  with_16(x, &u, &v);
  return fmaxf(u, v);
}
__device__ __forceinline__ float max_over_32(float x) {
  float u, v;
  with_32(x, &u, &v);
  return fmaxf(u, v);
}

// cos and sin of a (radians) in 64 bits.  a = n pi/2 + r, |r| <= pi/4, with pi/2 as the sum of
// three doubles (53 bits each, so that n pi/2 is exact far past n = 2^31), then the Taylor
// series of both to r^17 / r^16 (the next terms are below 2^-55 at pi/4).  About 35 instructions
// of the 64-bit unit; hipcc's sincos() takes a branch for large arguments that no position
// below 2^31 needs.
__device__ __forceinline__ void cos_sin(double a, double* c, double* s) {
  const double n = rint(a * 0.63661977236758134308);
  double r = fma(n, -1.57079632679489655800e+00, a);
  r = fma(n, -6.12323399573676603587e-17, r);
  r = fma(n, 1.49738490485916983028e-33, r);
  const double q = r * r;
  double ps = 1.0 / 355687428096000.0;  // 1 / 17!
  ps = fma(ps, q, -1.0 / 1307674368000.0);
  ps = fma(ps, q, 1.0 / 6227020800.0);
  ps = fma(ps, q, -1.0 / 39916800.0);
  ps = fma(ps, q, 1.0 / 362880.0);
  ps = fma(ps, q, -1.0 / 5040.0);
  ps = fma(ps, q, 1.0 / 120.0);
  ps = fma(ps, q, -1.0 / 6.0);
  const double sr = fma(ps * q, r, r);
  double pc = 1.0 / 20922789888000.0;  // 1 / 16!
  pc = fma(pc, q, -1.0 / 87178291200.0);
  pc = fma(pc, q, 1.0 / 479001600.0);
  pc = fma(pc, q, -1.0 / 3628800.0);
  pc = fma(pc, q, 1.0 / 40320.0);
  pc = fma(pc, q, -1.0 / 720.0);
  pc = fma(pc, q, 1.0 / 24.0);
  pc = fma(pc, q, -0.5);
  const double cr = fma(pc, q, 1.0);
  const int quarter = (int)(n - 4.0 * floor(n * 0.25));
  const double x = (quarter & 1) ? sr : cr, y = (quarter & 1) ? cr : sr;
  *c = (quarter == 1 || quarter == 2) ? -x : x;
  *s = quarter >= 2 ? -y : y;
}

// The factors of pair i at position p, rounded to 32 bits.  The angle is rounded once, to 64 bits.
__device__ __forceinline__ float2 rotation_of(const double* freq, double amplitude, int32_t p, int i) {
#pragma clang fp contract(off)
  const double angle = (double)p * freq[i];
  double c, s;
  cos_sin(angle, &c, &s);
  return make_float2((float)(c * amplitude), (float)(s * amplitude));
}

// One rotated pair.  Each operation is rounded (no fused multiply-add), so that a key is the same
// whichever kernel rotates it, and the block means made from keys are too.
__device__ __forceinline__ void rotate(float x0, float x1, float2 cs, float* y0, float* y1) {
#pragma clang fp contract(off)
  const float a = x0 * cs.x, b = x1 * cs.y, c = x1 * cs.x, d = x0 * cs.y;
  *y0 = a - b;
  *y1 = c + d;
}

}  // namespace
}  // namespace sdnn

#endif  // SDNN_DECODE_DEVICE_H_
