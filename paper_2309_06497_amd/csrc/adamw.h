// AdamW over all tensors of a model, and the norm of all gradients.
//
//   g <- g min(1, max_norm / norm)
//   m <- b1 m + (1 - b1) g        v <- b2 v + (1 - b2) g g        (each product and sum rounded to float32 by itself: the states of 8 bits that follow are
//   those of any float32 program that does the same steps)
//   p <- (1 - lr wd) p - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + epsilon)
//
// States in 8 bits: 128 neighbouring elements of a tensor share one byte, the exponent E of their largest (of m and of v).  A value 2^-E is kept as a number of
// 8 bits: m with a sign, 4 bits of exponent and 3 behind the first, v with 5 bits of exponent and 3: 14 (30) binades and, below them, multiples
// of the smallest value.  The largest lies one binade below the top, so that it can be rounded up.  v moves by a thousandth of itself in a step, far less
// than half a step of its code, so rounding to the nearest would keep it for ever; a code is rounded up with the probability of what is left over.
// The random numbers are a mix of the element's index and the step's number: the same call gives the same bits.  v > 0 is never rounded to zero: m over nothing
// but epsilon would be a leap.  Multiplied by 2^-113 (2^-97) the lowest binade becomes the lowest of float32, so that its own subnormal numbers are the code's, and a
// code is eight bits of a float32.
// bf16 parameters are rounded the same way: an update is mostly less than half a step of theirs.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include "group.h"
#include "vectors.h"

namespace shampoo {

constexpr int AW_GROUP = 128, AW_CHUNK = 4096, AW_TENSORS = 160;
constexpr uint32_t AW_MIX1 = 0x9E3779B9u, AW_MIX2 = 0x6A09E667u, AW_MIX3 = 0xBB67AE85u, AW_MIX4 = 0xA54FF53Bu;
constexpr uint32_t AW_EXP_NAN = 254, AW_EXP_ZERO = 27;         // groups from 2^127 on read NaN, below 2^-100 zero

// A piece of a tensor: where it begins there, among all elements, and among the 8-bit states (whose tensors begin with whole groups)
struct AdamChunk { int64_t start, flat, slot; int32_t len, tensor, decayed, unused; };

struct AdamState {
  float *m, *v;                                   // 32 bits: [all elements]
  uint8_t *m8, *v8, *m_exp, *v_exp;               // 8 bits: [slots], [slots / 128]
};
struct AdamArgs {
  const AdamChunk *chunks;
  AdamState state;
  const float *norm;                              // or nullptr
  float max_norm, b1, b1c, b2, b2c, inv_sqrt, epsilon, keep, lr;     // keep: 1 - lr wd; lr over the first correction, inv_sqrt: one over the root of the second
  uint32_t mix;                                   // of the step's number
  int32_t has_copies;
  void *p[AW_TENSORS]; const void *g[AW_TENSORS]; uint16_t *copy[AW_TENSORS];
};
static_assert(sizeof(AdamArgs) <= 4096, "arguments of a kernel");

// Products and sums that are rounded by themselves
__device__ __forceinline__ float product(float x, float y) {
#pragma clang fp contract(off)
  return x * y;
}
__device__ __forceinline__ float sum(float x, float y) {
#pragma clang fp contract(off)
  return x + y;
}

// 2^E and 2^-E of an exponent byte
__device__ __forceinline__ float exp_value(uint32_t byte) { return __uint_as_float(byte << 23); }
__device__ __forceinline__ float exp_inverse(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

// what a code (without sign) stands for, times 2^-E
template <int SHIFT> __device__ __forceinline__ float code_value(uint32_t code) { return __uint_as_float(code << 20) * __uint_as_float((uint32_t)(127 + SHIFT) << 23); }
template <int SHIFT> __device__ __forceinline__ uint32_t code_of(float magnitude, float inverse, uint32_t add) {
  return (__float_as_uint(magnitude * inverse * __uint_as_float((uint32_t)(127 - SHIFT) << 23)) + add) >> 20;
}
// eight neighbouring codes, the sign of m in bit 7
__device__ __forceinline__ void decode_m(uint2 q, uint32_t byte, f32x8 &x) {
  const float scale = byte == 255 ? NAN : exp_value(byte);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t c = ((e < 4 ? q.x : q.y) >> (8 * (e & 3))) & 255u;
    x.v[e] = __uint_as_float(__float_as_uint(code_value<113>(c & 127u) * scale) | (c >> 7) << 31);
  }
}
__device__ __forceinline__ void decode_v(uint2 q, uint32_t byte, f32x8 &x) {
  const float scale = byte == 255 ? NAN : exp_value(byte);
#pragma unroll
  for (int e = 0; e < 8; ++e) x.v[e] = code_value<97>(((e < 4 ? q.x : q.y) >> (8 * (e & 3))) & 255u) * scale;
}
// the exponent byte of a group, 16 lanes with eight values each
__device__ __forceinline__ uint32_t group_exponent(const f32x8 &x) {
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x.v[e]) & 0x7fffffffu);
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
  return top >> 23 >= AW_EXP_NAN ? 255u : top >> 23;
}
__device__ __forceinline__ uint2 encode_m(const f32x8 &x, uint32_t byte, const uint32_t (&add)[8]) {
  uint32_t w[2] = {0u, 0u};
  if (byte >= AW_EXP_ZERO && byte != 255) {
    const float inverse = exp_inverse(byte);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t u = __float_as_uint(x.v[e]), c = code_of<113>(fabsf(x.v[e]), inverse, add[e]) | (u >> 31) << 7;
      w[e >> 2] |= c << (8 * (e & 3));
    }
  }
  return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ uint2 encode_v(const f32x8 &x, uint32_t byte, const uint32_t (&add)[8]) {
  uint32_t w[2] = {0u, 0u};
  if (byte >= AW_EXP_ZERO && byte != 255) {
    const float inverse = exp_inverse(byte);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      uint32_t c = code_of<97>(fabsf(x.v[e]), inverse, add[e]);
      c = c == 0 && x.v[e] != 0.f ? 1u : c;
      w[e >> 2] |= c << (8 * (e & 3));
    }
  }
  return make_uint2(w[0], w[1]);
}

// Offsets of the roundings of element i in a step: of m and v in 2^-20, of a bf16 parameter in 2^-16
__device__ __forceinline__ void rounding_offsets(uint32_t seed, uint32_t &m, uint32_t &v, uint32_t &p) {
  uint32_t x = seed;
  x = (x ^ x >> 16) * AW_MIX3;
  x = (x ^ x >> 15) * AW_MIX4;
  x ^= x >> 16;
  uint32_t y = x * AW_MIX1 + AW_MIX2;
  y ^= y >> 15;
  m = x >> 12; v = y >> 12; p = y & 0xffffu;
}

// P, G: types of parameters and gradients (float or uint16_t, bf16 bits).  A thread has eight neighbouring elements.
template <typename P, typename G, int BITS> __global__ __launch_bounds__(256) void adamw_kernel(const AdamArgs g) {
  const AdamChunk c = g.chunks[blockIdx.x];
  float clip = 1.f;
  if (g.norm) {
    const float norm = *g.norm;
    if (!(fabsf(norm) < INFINITY)) return;                     // nothing is touched
    clip = norm > g.max_norm ? g.max_norm / norm : 1.f;
  }
  P *p = global_ptr<P>(g.p[c.tensor]) + c.start;
  const G *grad = global_ptr<const G>(g.g[c.tensor]) + c.start;
  uint16_t *copy = g.has_copies ? global_ptr<uint16_t>(g.copy[c.tensor]) + c.start : nullptr;
  const float keep = c.decayed ? g.keep : 1.f;
  for (int at = threadIdx.x * 8; at < ((c.len + AW_GROUP - 1) & ~(AW_GROUP - 1)); at += 2048) {
    const f32x8 x = load8(grad, at, c.len);
    f32x8 w = load8(p, at, c.len), m, v;
    if constexpr (BITS == 32) {
      m = load8(g.state.m + c.flat, at, c.len);
      v = load8(g.state.v + c.flat, at, c.len);
    } else {
      const int64_t s = c.slot + at;
      decode_m(*reinterpret_cast<const uint2 *>(g.state.m8 + s), g.state.m_exp[s / AW_GROUP], m);
      decode_v(*reinterpret_cast<const uint2 *>(g.state.v8 + s), g.state.v_exp[s / AW_GROUP], v);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float k = product(x.v[e], clip);
      m.v[e] = sum(product(m.v[e], g.b1), product(k, g.b1c));
      v.v[e] = sum(product(v.v[e], g.b2), product(product(k, g.b2c), k));
      const float u = m.v[e] / fmaf(sqrtf(v.v[e]), g.inv_sqrt, g.epsilon);
      w.v[e] = fmaf(-g.lr, u, w.v[e] * keep);
    }
    [[maybe_unused]] uint32_t rm[8], rv[8], rp[8];
    if constexpr (BITS == 8 || sizeof(P) == 2) {
      const uint64_t i = (uint64_t)c.flat + (uint32_t)at;       // eight neighbours may reach over 2^32
#pragma unroll
      for (int e = 0; e < 8; ++e) rounding_offsets((uint32_t)(i + e) * AW_MIX1 + (uint32_t)((i + e) >> 32) * AW_MIX3 + g.mix, rm[e], rv[e], rp[e]);
    }
    if constexpr (BITS == 32) {
      store8(g.state.m + c.flat, at, c.len, m);
      store8(g.state.v + c.flat, at, c.len, v);
    } else {
      const int64_t s = c.slot + at;
      const uint32_t em = group_exponent(m), ev = group_exponent(v);
      *reinterpret_cast<uint2 *>(g.state.m8 + s) = encode_m(m, em, rm);
      *reinterpret_cast<uint2 *>(g.state.v8 + s) = encode_v(v, ev, rv);
      if ((threadIdx.x & 15) == 0) { g.state.m_exp[s / AW_GROUP] = (uint8_t)em; g.state.v_exp[s / AW_GROUP] = (uint8_t)ev; }
    }
    if constexpr (sizeof(P) == 2) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t u = __float_as_uint(w.v[e]);
        // infinities and NaN as they are (a NaN keeps a bit)
        w.v[e] = __uint_as_float((u & 0x7f800000u) == 0x7f800000u ? (u & 0x7fffffu ? u | 0x400000u : u) & 0xffff0000u : (u + rp[e]) & 0xffff0000u);
      }
    }
    store8(p, at, c.len, w);
    if (copy) store8(copy, at, c.len, w);
  }
}

// States as values, one behind the other without gaps, or from there.
struct AdamValuesArgs { const AdamChunk *chunks; AdamState state; void *m, *v; };
template <typename T, int BITS> __global__ __launch_bounds__(256) void adamw_get_kernel(const AdamValuesArgs g) {
  const AdamChunk c = g.chunks[blockIdx.x];
  T *const to_m = static_cast<T *>(g.m) + c.flat, *const to_v = static_cast<T *>(g.v) + c.flat;
  for (int at = threadIdx.x * 8; at < c.len; at += 2048) {
    f32x8 m, v;
    if constexpr (BITS == 32) {
      m = load8(g.state.m + c.flat, at, c.len);
      v = load8(g.state.v + c.flat, at, c.len);
    } else {
      const int64_t s = c.slot + at;
      decode_m(*reinterpret_cast<const uint2 *>(g.state.m8 + s), g.state.m_exp[s / AW_GROUP], m);
      decode_v(*reinterpret_cast<const uint2 *>(g.state.v8 + s), g.state.v_exp[s / AW_GROUP], v);
    }
    store8(to_m, at, c.len, m);
    store8(to_v, at, c.len, v);
  }
}
// Codes to the nearest; m or v null: zeros.  A largest of just a power of two counts as the top of the binade below it, as which a step may have left it: what an
// optimizer held is held again.
__device__ __forceinline__ uint32_t loaded_exponent(const f32x8 &x) {
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x.v[e]) & 0x7fffffffu);
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
  const uint32_t byte = top >> 23 >= AW_EXP_NAN ? 255u : top >> 23;
  return byte != 255 && byte > AW_EXP_ZERO && (top & 0x7fffffu) == 0 ? byte - 1 : byte;
}
template <int BITS> __global__ __launch_bounds__(256) void adamw_set_kernel(const AdamValuesArgs g) {
  const AdamChunk c = g.chunks[blockIdx.x];
  const uint32_t half[8] = {0x80000u, 0x80000u, 0x80000u, 0x80000u, 0x80000u, 0x80000u, 0x80000u, 0x80000u};
  for (int at = threadIdx.x * 8; at < ((c.len + AW_GROUP - 1) & ~(AW_GROUP - 1)); at += 2048) {
    f32x8 m = {}, v = {};
    if (g.m) m = load8(static_cast<const float *>(g.m) + c.flat, at, c.len);
    if (g.v) v = load8(static_cast<const float *>(g.v) + c.flat, at, c.len);
    if constexpr (BITS == 32) {
      store8(g.state.m + c.flat, at, c.len, m);
      store8(g.state.v + c.flat, at, c.len, v);
    } else {
      const int64_t s = c.slot + at;
      const uint32_t em = loaded_exponent(m), ev = loaded_exponent(v);
      *reinterpret_cast<uint2 *>(g.state.m8 + s) = encode_m(m, em, half);
      *reinterpret_cast<uint2 *>(g.state.v8 + s) = encode_v(v, ev, half);
      if ((threadIdx.x & 15) == 0) { g.state.m_exp[s / AW_GROUP] = (uint8_t)em; g.state.v_exp[s / AW_GROUP] = (uint8_t)ev; }
    }
  }
}

// ---------------------------------------------------------------------------
// Norms: sums of squares in 64 bits (no float32 gradient's square leaves their range), one per piece of a tensor, added up in order.
// ---------------------------------------------------------------------------
constexpr int GN_TENSORS = 192;
struct NormArgs {
  double *part; int32_t *first;                   // sums of pieces; first[t]: the first of tensor t, one more behind the last
  int32_t tensors, tensor0, block0, blocks;       // of this launch; block0: its first piece
  int32_t chunk;                                  // elements of a piece
  int32_t at[GN_TENSORS];                         // first piece of a tensor, counted from block0
  const void *g[GN_TENSORS]; int64_t len[GN_TENSORS];
};
static_assert(sizeof(NormArgs) <= 4096, "arguments of a kernel");
__device__ __forceinline__ double sum_256(double s) {
  __shared__ double part[4];
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) s += __shfl_xor(s, o, 64);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
  __syncthreads();
  return (part[0] + part[1]) + (part[2] + part[3]);
}
template <typename G> __global__ __launch_bounds__(256) void square_sums_kernel(const NormArgs g) {
  const int block = blockIdx.x;
  if (block == 0) {
    for (int t = threadIdx.x; t < g.tensors; t += 256) g.first[g.tensor0 + t] = g.block0 + g.at[t];
    if (threadIdx.x == 0) g.first[g.tensor0 + g.tensors] = g.block0 + g.blocks;
  }
  if (block >= g.blocks) return;
  int lo = 0, hi = g.tensors;                     // the last tensor that begins here or before: empty ones end where they begin
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (g.at[mid] <= block) lo = mid; else hi = mid;
  }
  const int64_t start = (int64_t)(block - g.at[lo]) * g.chunk;
  const G *x = global_ptr<const G>(g.g[lo]) + start;
  const int n = (int)min((int64_t)g.chunk, g.len[lo] - start);
  double s = 0.0;
  for (int c = threadIdx.x * 8; c < n; c += 2048) {
    const f32x8 v = load8(x, c, n);
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fma((double)v.v[e], (double)v.v[e], s);
  }
  s = sum_256(s);
  if (threadIdx.x == 0) g.part[g.block0 + block] = s;
}
// a workgroup per tensor, and the last one for all
__global__ __launch_bounds__(256) void norms_kernel(const double *part, const int32_t *first, int32_t tensors, float *norm, float *norms) {
  const int t = blockIdx.x;
  const int from = t < tensors ? first[t] : 0, to = t < tensors ? first[t + 1] : first[tensors];
  double s = 0.0;
  for (int i = from + threadIdx.x; i < to; i += 256) s += part[i];
  s = sum_256(s);
  if (threadIdx.x != 0) return;
  if (t < tensors) { if (norms) norms[t] = (float)sqrt(s); }
  else *norm = (float)sqrt(s);
}

}  // namespace shampoo
