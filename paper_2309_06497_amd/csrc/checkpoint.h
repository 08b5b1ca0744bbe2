// Activation checkpoints in 8 bits.
//
// A matrix [rows][cols] is kept as codes q (int8) and one exponent s per row and group of 32 neighbouring features:
// x ~ q 2^s, q = rint(x 2^-s), with the smallest s for which the group's largest |x| rounds to at most 127.  A power of two
// for the scale makes every step of both directions exact but the one rounding (x 2^-s is exact, q 2^s is a bf16 value), so
// that the products that read a checkpoint (train_gemm.h) lose nothing more, and the codes do not depend on how a
// kernel orders its work.  The error of an element is at most half a step: 1/255 ... 1/127.5 of the largest of its group.
// Groups whose largest element is below 2^-100 are zero; a group with an infinity, a NaN or an element from 255 2^120
// on is NaN as a whole.
//
// In memory: codes [rows][pitch], pitch = cols rounded up to 32 (zeros at the end of a row), then, from the next multiple of
// 256 bytes on, the exponents [rows][pitch / 32], one byte each: s + 133 (0: zero group, 255: not finite).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include "vectors.h"

namespace shampoo {

enum { ACT_NONE = 0, ACT_RELU = 1, ACT_GELU = 2, ACT_SILU = 3 };

struct Packed {
  int8_t *codes; uint8_t *exps;
  int64_t rows;
  int32_t cols, pitch;
};

// The exponent byte of a group from the bits of its largest |x|: x in [1, 2) 2^e gives s = e - 6, or e - 5 where x 2^(6 - e)
// would round to 128 (from 127.5 on: the upper seven mantissa bits all ones, which the addition carries into the exponent).
__device__ __forceinline__ uint32_t exponent_byte(uint32_t largest) {
  if (largest >= 0x7f7f0000u) return 255u;                  // would carry into the exponent of infinity
  if (largest < (27u << 23)) return 0u;                     // 2^-100
  return (largest + 0x10000u) >> 23;                        // e + 127 = s + 133
}
// 2^-s and 2^s of an exponent byte (27 ... 254); for byte 0 the codes are zero, for 255 the scale makes them NaN
__device__ __forceinline__ float code_per_value(uint32_t byte) { return __uint_as_float((260u - min(max(byte, 27u), 254u)) << 23); }
__device__ __forceinline__ float value_per_code(uint32_t byte) {
  return byte == 255u ? __uint_as_float(0x7fc00000u) : byte < 27u ? 0.f : __uint_as_float((byte - 6u) << 23);
}

// Eight neighbouring values of a lane, four neighbouring lanes a group: their codes, and the group's byte in `byte`.  Beside
// 1.5 2^23 the unit of a float32 is 1: adding that rounds x 2^-s to even and leaves the code in the low byte.
__device__ __forceinline__ uint2 pack8(const f32x8 &x, uint32_t &byte) {
  uint32_t largest = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) largest = max(largest, __float_as_uint(x.v[e]) & 0x7fffffffu);
  largest = max(largest, (uint32_t)__shfl_xor((int)largest, 1, 64));
  largest = max(largest, (uint32_t)__shfl_xor((int)largest, 2, 64));
  byte = exponent_byte(largest);
  const float per = code_per_value(byte);
  uint32_t q[8], w[2];
#pragma unroll
  for (int e = 0; e < 8; ++e) q[e] = __float_as_uint(fmaf(x.v[e], per, 12582912.f));
#pragma unroll
  for (int h = 0; h < 2; ++h)                                // the low bytes of four, first one lowest
    w[h] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(q[4 * h + 3], q[4 * h + 2], 0x0c0c0400u), __builtin_amdgcn_perm(q[4 * h + 1], q[4 * h], 0x0c0c0400u), 0x05040100u);
  if (byte == 0u) w[0] = w[1] = 0u;
  if (byte == 255u) w[0] = w[1] = 0x01010101u;               // 1 x NaN
  return make_uint2(w[0], w[1]);
}
// from q + 128, which a conversion takes out of its word (128 2^s itself may be past float32)
__device__ __forceinline__ f32x8 unpack8(uint2 w, float scale) {
  f32x8 r;
  const uint32_t u[2] = {w.x ^ 0x80808080u, w.y ^ 0x80808080u};
#pragma unroll
  for (int e = 0; e < 8; ++e) r.v[e] = ((float)((u[e >> 2] >> (8 * (e & 3))) & 255u) - 128.f) * scale;
  return r;
}
// eight values at column c (a multiple of 8 below pitch) of row i
__device__ __forceinline__ f32x8 packed_load8(const Packed &p, int64_t i, int c) {
  const uint2 w = *reinterpret_cast<const uint2 *>(p.codes + i * p.pitch + c);
  return unpack8(w, value_per_code(p.exps[i * (p.pitch >> 5) + (c >> 5)]));
}
// all 64 lanes have to take part; lanes past the row's end with zeros
__device__ __forceinline__ void packed_store8(const Packed &p, int64_t i, int c, const f32x8 &x) {
  uint32_t byte;
  const uint2 w = pack8(x, byte);
  if (c >= p.pitch) return;
  *reinterpret_cast<uint2 *>(p.codes + i * p.pitch + c) = w;
  if ((c & 31) == 0) p.exps[i * (p.pitch >> 5) + (c >> 5)] = (uint8_t)byte;
}

// a(z) and a'(z) of eight values.  The choice lies outside the loops: a wavefront fetches the code of one function only.
template <typename F> __device__ __forceinline__ void each8(f32x8 &z, F &&f) {
#pragma unroll
  for (int e = 0; e < 8; ++e) z.v[e] = f(z.v[e]);
}
__device__ __forceinline__ void activate8(f32x8 &z, int kind) {
  switch (kind) {
    case ACT_RELU: each8(z, [](float x) { return x > 0.f ? x : x != x ? x : 0.f; }); break;
    case ACT_GELU: each8(z, [](float x) { return 0.5f * x * (1.f + erff(x * 0.70710678118654752f)); }); break;
    case ACT_SILU: each8(z, [](float x) { return x / (1.f + expf(-x)); }); break;
    default: break;
  }
}
__device__ __forceinline__ void slope8(f32x8 &z, int kind) {
  switch (kind) {
    case ACT_RELU: each8(z, [](float x) { return x > 0.f ? 1.f : x != x ? x : 0.f; }); break;
    case ACT_GELU: each8(z, [](float x) { return 0.5f * (1.f + erff(x * 0.70710678118654752f)) + x * expf(-0.5f * x * x) * 0.39894228040143268f; }); break;
    case ACT_SILU: each8(z, [](float x) { const float s = 1.f / (1.f + expf(-x)); return s * (1.f + x * (1.f - s)); }); break;
    default: each8(z, [](float) { return 1.f; });
  }
}

// Pieces of eight in row order: a thread takes one piece, a grid at most 2^30 of them; row0: the grid's first row.
// One pass, 16 bytes (8 for codes) per lane: bound by memory.  8192 x 8192 in bf16: packed in 39 us, read back in 33 (203 MB each,
// 5.2 and 6.2 TB/s, part of it from the cache behind the L2); the GELU gradient of 3001 x 4001 in float32 22 us (108 MB, 4.9 TB/s).
struct PackArgs {
  const void *x; int64_t ldx;
  Packed p;
  int64_t row0; uint32_t pieces, per_row;      // pieces of this grid; pitch / 8
};
template <typename T> __global__ __launch_bounds__(256) void checkpoint_pack_kernel(const PackArgs g) {
  const uint32_t i = blockIdx.x * 256u + threadIdx.x;
  const uint32_t r = min(i, g.pieces - 1) / g.per_row;
  const int c = (int)(min(i, g.pieces - 1) - r * g.per_row) * 8;
  const int64_t row = g.row0 + r;
  const f32x8 x = load8(static_cast<const T *>(g.x) + row * g.ldx, c, g.p.cols);
  uint32_t byte;
  const uint2 w = pack8(x, byte);                // per_row is a multiple of 4: a group never straddles rows or wavefronts
  if (i >= g.pieces) return;
  *reinterpret_cast<uint2 *>(g.p.codes + row * g.p.pitch + c) = w;
  if ((c & 31) == 0) g.p.exps[row * (g.p.pitch >> 5) + (c >> 5)] = (uint8_t)byte;
}

// y = a(x), or dx = dy a'(x)
struct UnpackArgs {
  Packed p;
  const void *dy; int64_t lddy;                // GRAD
  void *y; int64_t ldy;
  int64_t row0; uint32_t pieces, per_row;
  int32_t activation;
};
template <typename T, bool GRAD> __global__ __launch_bounds__(256) void checkpoint_unpack_kernel(const UnpackArgs g) {
  const uint32_t i = blockIdx.x * 256u + threadIdx.x;
  if (i >= g.pieces) return;
  const uint32_t r = i / g.per_row;
  const int c = (int)(i - r * g.per_row) * 8;
  const int64_t row = g.row0 + r;
  if (c >= g.p.cols) return;
  f32x8 x = packed_load8(g.p, row, c);
  if constexpr (GRAD) {
    const f32x8 d = load8(static_cast<const T *>(g.dy) + row * g.lddy, c, g.p.cols);
    slope8(x, g.activation);
#pragma unroll
    for (int e = 0; e < 8; ++e) x.v[e] *= d.v[e];
  } else {
    activate8(x, g.activation);
  }
  store8(static_cast<T *>(g.y) + row * g.ldy, c, g.p.cols, x);
}

// a(x) of a checkpoint, or a matrix in memory (float32 or bf16, any alignment), as PLANES bf16 planes [plane][rows][ld], ld a
// multiple of 8, zeros from cols to ld and in rows from `rows` on.  Bound by memory: one plane of 8192 x 8192 codes 37 us (5.5 TB/s).
struct PlanesArgs {
  Packed p; const void *x; int64_t ldx;        // one of the two
  uint16_t *out; int64_t plane, ld;
  int64_t rows, row0; uint32_t pieces, per_row;      // ld / 8
  int32_t cols, activation;
};
enum { FROM_PACKED = 0, FROM_F32 = 1, FROM_BF16 = 2 };
template <int FROM, int PLANES> __device__ __forceinline__ void planes_piece(const PlanesArgs &g, uint32_t i) {
  if (i >= g.pieces) return;
  const uint32_t r = i / g.per_row;
  const int c = (int)(i - r * g.per_row) * 8;
  const int64_t row = g.row0 + r;
  f32x8 x = {{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}};
  if (row >= g.rows) {
  } else if constexpr (FROM == FROM_PACKED) {
    if (c < g.p.pitch) x = packed_load8(g.p, row, c);
    activate8(x, g.activation);
    if (c + 8 > g.cols) {                          // a group that is not finite reads NaN in the padding too
#pragma unroll
      for (int e = 0; e < 8; ++e) if (c + e >= g.cols) x.v[e] = 0.f;
    }
  } else if constexpr (FROM == FROM_F32) {
    x = load8(static_cast<const float *>(g.x) + row * g.ldx, c, g.cols);
  } else {
    x = load8(static_cast<const uint16_t *>(g.x) + row * g.ldx, c, g.cols);
  }
  uint16_t q[8][PLANES];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if constexpr (FROM == FROM_F32) bf16_planes_of_any(x.v[e], q[e]); else bf16_planes_of<PLANES>(x.v[e], q[e]);
  }
#pragma unroll
  for (int t = 0; t < PLANES; ++t) {
    uint4 w;
    w.x = q[0][t] | (uint32_t)q[1][t] << 16; w.y = q[2][t] | (uint32_t)q[3][t] << 16;
    w.z = q[4][t] | (uint32_t)q[5][t] << 16; w.w = q[6][t] | (uint32_t)q[7][t] << 16;
    *reinterpret_cast<uint4 *>(g.out + t * g.plane + row * g.ld + c) = w;
  }
}
// Column sums of x (float32 or bf16) by parts of its rows, in an order that does not depend on the launch: 64 columns of one part a
// workgroup, four threads a column.  They go along with the planes of a product's operands: a launch of their own took 4 us.
struct ColumnSumsArgs { const void *x; int64_t ldx, rows, per_part; float *out; int32_t cols, bf16; };      // out: [parts][cols]
__device__ __forceinline__ void column_sums(const ColumnSumsArgs &g, uint32_t block) {
  __shared__ float part[4][64];
  const uint32_t across = (uint32_t)(g.cols + 63) / 64, p = block / across;
  const int c = threadIdx.x & 63, k = threadIdx.x >> 6, j = (int)(block - p * across) * 64 + c;
  const int64_t i0 = p * g.per_part, i1 = min(g.rows, i0 + g.per_part);
  auto rows = [&](auto value) {
    float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    int64_t i = i0 + k;
    for (; i + 28 < i1; i += 32) {
#pragma unroll
      for (int q = 0; q < 8; ++q) s[q] += value(i + 4 * q);
    }
    for (; i < i1; i += 4) s[0] += value(i);
    return ((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7]));
  };
  float s = 0.f;
  if (j < g.cols) {
    if (g.bf16) s = rows([&](int64_t i) { return bf16_value(static_cast<const uint16_t *>(g.x)[i * g.ldx + j]); });
    else s = rows([&](int64_t i) { return static_cast<const float *>(g.x)[i * g.ldx + j]; });
  }
  part[k][c] = s;
  __syncthreads();
  if (k == 0 && j < g.cols) g.out[(int64_t)p * g.cols + j] = (part[0][c] + part[1][c]) + (part[2][c] + part[3][c]);
}

// SUMS: workgroups from `blocks` on have column sums.
template <int FROM, int PLANES, bool SUMS>
__global__ __launch_bounds__(256) void planes_kernel(const PlanesArgs g, uint32_t blocks, const ColumnSumsArgs sums) {
  if (SUMS && blockIdx.x >= blocks) column_sums(sums, blockIdx.x - blocks);
  else planes_piece<FROM, PLANES>(g, blockIdx.x * 256u + threadIdx.x);
}
// Both operands of a product in one launch: the first `blocks` workgroups have g, those up to `sums_from` h.
template <int FROM_G, int PLANES_G, int FROM_H, int PLANES_H>
__global__ __launch_bounds__(256) void planes_pair_kernel(const PlanesArgs g, const PlanesArgs h, uint32_t blocks, uint32_t sums_from, const ColumnSumsArgs sums) {
  if (blockIdx.x < blocks) planes_piece<FROM_G, PLANES_G>(g, blockIdx.x * 256u + threadIdx.x);
  else if (blockIdx.x < sums_from) planes_piece<FROM_H, PLANES_H>(h, (blockIdx.x - blocks) * 256u + threadIdx.x);
  else column_sums(sums, blockIdx.x - sums_from);
}

}  // namespace shampoo
