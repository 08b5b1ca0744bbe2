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

// Elements c ... c + 7 of a row of n, zeros past its end.  vec: the row starts on a multiple of 16 bytes (c % 8 == 0), so that
// a whole piece is read or written 16 bytes at a time.
template <typename T> __device__ __forceinline__ f32x8 load8(const T *row, int c, int n, bool vec) {
  f32x8 r;
  if (vec && c + 8 <= n) {
    if constexpr (sizeof(T) == 4) {
      const float4 a = *reinterpret_cast<const float4 *>(row + c), b = *reinterpret_cast<const float4 *>(row + c + 4);
      r = {{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
    } else {
      const uint4 u = *reinterpret_cast<const uint4 *>(row + c);
      const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) { r.v[2 * e] = __uint_as_float(w[e] << 16); r.v[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u); }
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      r.v[e] = 0.f;
      if (c + e < n) { if constexpr (sizeof(T) == 4) r.v[e] = row[c + e]; else r.v[e] = bf16_value(row[c + e]); }
    }
  }
  return r;
}
template <typename T> __device__ __forceinline__ void store8(T *row, int c, int n, bool vec, const f32x8 &x) {
  if (vec && c + 8 <= n) {
    if constexpr (sizeof(T) == 4) {
      *reinterpret_cast<float4 *>(row + c) = make_float4(x.v[0], x.v[1], x.v[2], x.v[3]);
      *reinterpret_cast<float4 *>(row + c + 4) = make_float4(x.v[4], x.v[5], x.v[6], x.v[7]);
    } else {
      *reinterpret_cast<uint4 *>(row + c) = make_uint4(bf16_pair(x.v[0], x.v[1]), bf16_pair(x.v[2], x.v[3]),
                                                       bf16_pair(x.v[4], x.v[5]), bf16_pair(x.v[6], x.v[7]));
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (c + e < n) { if constexpr (sizeof(T) == 4) row[c + e] = x.v[e]; else row[c + e] = bf16_bits(x.v[e]); }
  }
}

// x = sum of planes, each bf16: the first rounds x, the others what that leaves (three hold all 24 bits)
template <int PLANES> __device__ __forceinline__ void bf16_planes_of(float x, uint16_t (&p)[PLANES]) {
#pragma unroll
  for (int t = 0; t < PLANES; ++t) {
    p[t] = bf16_bits(x);
    if (t + 1 < PLANES) x -= bf16_value(p[t]);
  }
}

}  // namespace shampoo
