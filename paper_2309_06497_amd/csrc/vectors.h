// Rows of float32 or bf16 values in pieces of eight, for the elementwise training kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include "lds_dma.h"

namespace shampoo {

struct f32x8 { float v[8]; };

__device__ __forceinline__ float bf16_value(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }
__device__ __forceinline__ uint16_t bf16_bits(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }
__device__ __forceinline__ uint32_t bf16_pair(float x, float y) {
  typedef float pair __attribute__((ext_vector_type(2)));
  typedef __bf16 bpair __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(pair{x, y}, bpair));
}

// Rows may start at any multiple of their element: the memory takes 16-byte accesses that are not aligned (a row that is costs
// a cache line less per 64 lanes).
typedef uint32_t rows_u32x4 __attribute__((ext_vector_type(4)));
template <typename T> struct RowVector;
template <> struct RowVector<float> { typedef rows_u32x4 type __attribute__((aligned(4))); };
template <> struct RowVector<uint16_t> { typedef rows_u32x4 type __attribute__((aligned(2))); };

// Elements c ... c + 7 of a row of n as they are in memory, zeros past its end.
template <typename T> struct Raw8 { rows_u32x4 u[sizeof(T) / 2]; };
template <typename T> __device__ __forceinline__ Raw8<T> raw_load8(const T *row, int c, int n) {
  Raw8<T> r;
  if (c + 8 <= n) {
#pragma unroll
    for (int k = 0; k < (int)sizeof(T) / 2; ++k) r.u[k] = reinterpret_cast<const typename RowVector<T>::type *>(row + c)[k];
  } else {
#pragma unroll
    for (int k = 0; k < (int)sizeof(T) / 2; ++k) r.u[k] = rows_u32x4{0u, 0u, 0u, 0u};
    if (c < n) {
#pragma unroll
      for (int e = 0; e < 7; ++e)
        if (c + e < n) {
          if constexpr (sizeof(T) == 4) r.u[e >> 2][e & 3] = __float_as_uint(row[c + e]);
          else r.u[0][e >> 1] |= (uint32_t)row[c + e] << (16 * (e & 1));
        }
    }
  }
  return r;
}
template <typename T> __device__ __forceinline__ f32x8 expand8(const Raw8<T> &r) {
  f32x8 x;
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x.v[e] = __uint_as_float(r.u[e >> 2][e & 3]);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) { x.v[2 * e] = __uint_as_float(r.u[0][e] << 16); x.v[2 * e + 1] = __uint_as_float(r.u[0][e] & 0xffff0000u); }
  }
  return x;
}
template <typename T> __device__ __forceinline__ f32x8 load8(const T *row, int c, int n) { return expand8(raw_load8(row, c, n)); }
template <typename T> __device__ __forceinline__ void store8(T *row, int c, int n, const f32x8 &x) {
  if (c + 8 <= n) {
#pragma unroll
    for (int k = 0; k < (int)sizeof(T) / 2; ++k) {
      rows_u32x4 u;
#pragma unroll
      for (int e = 0; e < 4; ++e) { if constexpr (sizeof(T) == 4) u[e] = __float_as_uint(x.v[4 * k + e]); else u[e] = bf16_pair(x.v[2 * e], x.v[2 * e + 1]); }
      reinterpret_cast<typename RowVector<T>::type *>(row + c)[k] = u;
    }
  } else if (c < n) {
#pragma unroll
    for (int e = 0; e < 7; ++e)
      if (c + e < n) { if constexpr (sizeof(T) == 4) row[c + e] = x.v[e]; else row[c + e] = bf16_bits(x.v[e]); }
  }
}

// x = sum of planes, each bf16: the first rounds x, the others what that leaves (three hold all 24 bits).  |x| < 3.396e38, from where on
// bf16 rounds to infinity.
template <int PLANES> __device__ __forceinline__ void bf16_planes_of(float x, uint16_t (&p)[PLANES]) {
#pragma unroll
  for (int t = 0; t < PLANES; ++t) {
    p[t] = bf16_bits(x);
    if (t + 1 < PLANES) x -= bf16_value(p[t]);
  }
}

// The same of any float32.  The largest ones begin with bf16's largest.  An infinity is the third plane, behind a one of its sign: it meets the
// other operand's first plane alone (plane_pairs), so that a product is infinite with the sign of the two, where infinity in the first plane would meet
// zeros, and second planes of either sign.
__device__ __forceinline__ void bf16_planes_of_any(float x, uint16_t (&p)[3]) {
  constexpr float MOST = 3.3895313892515355e38f;
  const bool infinite = fabsf(x) == INFINITY;
  float rest = infinite ? copysignf(1.f, x) : x;
  p[0] = bf16_bits(fminf(fmaxf(rest, -MOST), MOST));
  rest -= bf16_value(p[0]);                        // NaN: there from here on
  p[1] = bf16_bits(rest);
  p[2] = bf16_bits(infinite ? x : rest - bf16_value(p[1]));
}

}  // namespace shampoo
