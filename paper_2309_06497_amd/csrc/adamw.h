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

constexpr int AW_GROUP = 128, AW_CHUNK = 2048, AW_POINTERS = 480;       // of a launch: 240 tensors, 160 with copies
constexpr uint32_t AW_MIX1 = 0x9E3779B9u, AW_MIX2 = 0x6A09E667u, AW_MIX3 = 0xBB67AE85u, AW_MIX4 = 0xA54FF53Bu;
constexpr uint32_t AW_EXP_NAN = 254, AW_EXP_ZERO = 27;         // groups from 2^127 on read NaN, below 2^-100 zero

// A piece of a tensor: where it begins there, among all elements, and among the 8-bit states (whose tensors begin with whole groups)
struct AdamChunk { int64_t start, flat, slot; int32_t len, tensor, decayed, unused; };

// and what it is made from: first: the tensor's first piece
struct AdamTensor { int64_t first, numel, flat, slot; int32_t decayed, unused; };
__global__ __launch_bounds__(256) void adamw_chunks_kernel(const AdamTensor *tensors, int32_t n, AdamChunk *chunks, int64_t count) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= count) return;
  int lo = 0, hi = n;                             // the last tensor that begins here or before: empty ones begin where the next one does
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (tensors[mid].first <= i) lo = mid; else hi = mid;
  }
  const AdamTensor t = tensors[lo];
  const int64_t at = (i - t.first) * AW_CHUNK;
  chunks[i] = {at, t.flat + at, t.slot + at, (int32_t)min((int64_t)AW_CHUNK, t.numel - at), lo, t.decayed, 0};
}

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
  int32_t tensor0, tensors, has_copies;
  const void *tensor[AW_POINTERS];                // parameters, gradients, copies
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

// Eight neighbouring codes of a group whose exponent byte is `byte`, and back; the sign of m in bit 7.  A code's bits, 20 places up, are those of a float32 that is
// 2^-(SHIFT + E) of the value; scaling by that power of two is one exact instruction (and one rounding, of what is below the lowest binade's last bit but 20).
constexpr int AW_SHIFT_M = 113, AW_SHIFT_V = 97;
__device__ __forceinline__ void decode_m(uint2 q, uint32_t byte, f32x8 &x) {
  const int power = (int)byte - 127 + AW_SHIFT_M;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t c = (e < 4 ? q.x : q.y) << (24 - 8 * (e & 3));
    x.v[e] = __builtin_amdgcn_ldexpf(__uint_as_float((c >> 4 & 0x07f00000u) | (c & 0x80000000u)), power);
  }
  if (__any(byte == 255)) {                // hardly ever
#pragma unroll
    for (int e = 0; e < 8; ++e) x.v[e] = byte == 255 ? NAN : x.v[e];
  }
}
__device__ __forceinline__ void decode_v(uint2 q, uint32_t byte, f32x8 &x) {
  const int power = (int)byte - 127 + AW_SHIFT_V;
#pragma unroll
  for (int e = 0; e < 8; ++e) x.v[e] = __builtin_amdgcn_ldexpf(__uint_as_float(((e < 4 ? q.x : q.y) >> (8 * (e & 3)) & 255u) << 20), power);
  if (__any(byte == 255)) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x.v[e] = byte == 255 ? NAN : x.v[e];
  }
}
// Bits of the largest magnitude of a group, 16 lanes with eight values each
__device__ __forceinline__ uint32_t group_largest(const f32x8 &x) {
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 8; e += 2) top = max(top, max(__float_as_uint(x.v[e]) & 0x7fffffffu, __float_as_uint(x.v[e + 1]) & 0x7fffffffu));
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
  return top;
}
// its exponent byte
__device__ __forceinline__ uint32_t group_exponent(const f32x8 &x) {
  const uint32_t byte = group_largest(x) >> 23;
  return byte >= AW_EXP_NAN ? 255u : byte;
}
__device__ __forceinline__ uint2 encode_m(const f32x8 &x, uint32_t byte, const uint32_t (&add)[8]) {
  uint32_t w[2] = {0u, 0u};
  const int power = 127 - AW_SHIFT_M - (int)byte;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t c = (__float_as_uint(__builtin_amdgcn_ldexpf(fabsf(x.v[e]), power)) + add[e]) >> 20;
    w[e >> 2] |= (c | (__float_as_uint(x.v[e]) >> 24 & 128u)) << (8 * (e & 3));
  }
  const bool some = byte >= AW_EXP_ZERO && byte != 255;
  return make_uint2(some ? w[0] : 0u, some ? w[1] : 0u);
}
__device__ __forceinline__ uint2 encode_v(const f32x8 &x, uint32_t byte, const uint32_t (&add)[8]) {
  uint32_t w[2] = {0u, 0u};
  const int power = 127 - AW_SHIFT_V - (int)byte;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float v = fabsf(x.v[e]);
    const uint32_t c = (__float_as_uint(__builtin_amdgcn_ldexpf(v, power)) + add[e]) >> 20;
    w[e >> 2] |= max(c, min(__float_as_uint(v), 1u)) << (8 * (e & 3));        // only zero is zero
  }
  const bool some = byte >= AW_EXP_ZERO && byte != 255;
  return make_uint2(some ? w[0] : 0u, some ? w[1] : 0u);
}

// Offsets of the roundings of elements i ... i + 7 in a step: of m and v in 2^-20, of a bf16 parameter in 2^-16
__device__ __forceinline__ void rounding_offsets(uint64_t i, uint32_t mix, uint32_t (&m)[8], uint32_t (&v)[8], uint32_t (&p)[8]) {
  const uint32_t low = (uint32_t)i, seed = low * AW_MIX1 + (uint32_t)(i >> 32) * AW_MIX3 + mix;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    uint32_t x = seed + (uint32_t)e * AW_MIX1;
    if (low > 0xfffffff8u && low + e < low) x += AW_MIX3;      // over 2^32
    x = (x ^ x >> 16) * AW_MIX3;
    x = (x ^ x >> 15) * AW_MIX4;
    x ^= x >> 16;
    uint32_t y = x * AW_MIX1 + AW_MIX2;
    y ^= y >> 15;
    m[e] = x >> 12; v[e] = y >> 12; p[e] = y & 0xffffu;
  }
}

// P, G: types of parameters and gradients (float or uint16_t, bf16 bits).  A thread has eight neighbouring elements, a workgroup 2048 (4096 and 8192: 4 and 5 % longer with float32
// parameters).  Bound by memory: 200 M float32 parameters with bf16 gradients and copies, 32 bits 1.03 ms (28 bytes each, 5.4 TB/s), 671 M with 8 bits 1.99 ms (16 bytes, 5.4 TB/s);
// bf16 parameters with 8 bits (10 bytes) by 72 vector operations an element, three of them products of 32 bits for the random numbers: 67 M in 160 us, 4.2 TB/s.
template <typename P, typename G, int BITS> __global__ __launch_bounds__(256) void adamw_kernel(const AdamArgs g) {
  const AdamChunk c = g.chunks[blockIdx.x];
  float clip = 1.f;
  if (g.norm) {
    const float norm = *g.norm;
    if (!(fabsf(norm) < INFINITY)) return;                     // nothing is touched
    clip = norm > g.max_norm ? g.max_norm / norm : 1.f;
  }
  const int t = c.tensor - g.tensor0;
  P *p = global_ptr<P>(g.tensor[t]) + c.start;
  const G *grad = global_ptr<const G>(g.tensor[g.tensors + t]) + c.start;
  uint16_t *copy = g.has_copies ? global_ptr<uint16_t>(g.tensor[2 * g.tensors + t]) + c.start : nullptr;
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
      // root and reciprocal of the GPU's instructions: within one step; a v below 1.2e-38 has the root 0, not 1.1e-19 or less: epsilon is 1e-12 at least
      const float u = m.v[e] * __builtin_amdgcn_rcpf(fmaf(__builtin_amdgcn_sqrtf(v.v[e]), g.inv_sqrt, g.epsilon));
      w.v[e] = fmaf(-g.lr, u, w.v[e] * keep);
    }
    [[maybe_unused]] uint32_t rm[8], rv[8], rp[8];
    if constexpr (BITS == 8 || sizeof(P) == 2) {
      rounding_offsets((uint64_t)c.flat + (uint32_t)at, g.mix, rm, rv, rp);
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
        const float up = __uint_as_float((__float_as_uint(w.v[e]) + rp[e]) & 0xffff0000u);      // an infinity stays one
        w.v[e] = w.v[e] != w.v[e] ? NAN : up;
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
  const uint32_t top = group_largest(x), byte = top >> 23 >= AW_EXP_NAN ? 255u : top >> 23;
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
// Norms: sums of squares in 64 bits (no float32 gradient's square leaves their range), one per piece of a tensor, added up in order.  Bound by memory: 671 M bf16 gradients 222 us,
// 6.0 TB/s, four loads of a thread on their way together (one: 273).
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
template <int THREADS> __device__ __forceinline__ double sum_of(double s) {
  __shared__ double part[THREADS / 64];
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) s += __shfl_xor(s, o, 64);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
  __syncthreads();
  s = part[0];
#pragma unroll
  for (int k = 1; k < THREADS / 64; ++k) s += part[k];
  return s;
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
  constexpr int AHEAD = 4;
  double part[AHEAD] = {0.0, 0.0, 0.0, 0.0};
  const auto add = [](double &s, const f32x8 &v) {
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fma((double)v.v[e], (double)v.v[e], s);
  };
  int c = threadIdx.x * 8;
  for (; c + (AHEAD - 1) * 2048 + 8 <= n; c += AHEAD * 2048) {
    Raw8<G> raw[AHEAD];
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) raw[a] = raw_load8(x, c + a * 2048, 0x7fffffff);
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) add(part[a], expand8(raw[a]));
  }
  for (; c < n; c += 2048) add(part[0], load8(x, c, n));
  const double s = sum_of<256>((part[0] + part[1]) + (part[2] + part[3]));
  if (threadIdx.x == 0) g.part[g.block0 + block] = s;
}
// a workgroup per tensor, and the last one for all
__global__ __launch_bounds__(1024) void norms_kernel(const double *part, const int32_t *first, int32_t tensors, float *norm, float *norms) {
  const int t = blockIdx.x;
  const int from = t < tensors ? first[t] : 0, to = t < tensors ? first[t + 1] : first[tensors];
  double s[4] = {0.0, 0.0, 0.0, 0.0};
  int i = from + (int)threadIdx.x;
  for (; i + 3 * 1024 < to; i += 4 * 1024) {
#pragma unroll
    for (int a = 0; a < 4; ++a) s[a] += part[i + a * 1024];
  }
  for (; i < to; i += 1024) s[0] += part[i];
  const double all = sum_of<1024>((s[0] + s[1]) + (s[2] + s[3]));
  if (threadIdx.x != 0) return;
  if (t < tensors) { if (norms) norms[t] = (float)sqrt(all); }
  else *norm = (float)sqrt(all);
}

}  // namespace shampoo
