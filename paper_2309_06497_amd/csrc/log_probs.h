// Log probabilities of given tokens, entropies and most probable tokens from logits z, and the gradient of the logits.
//
//   x_v = (z_v - m) / T        m = max z        s = sum_v exp x_v
//   log p_v = x_v - log s        H = -sum p_v log p_v = log s - sum_v x_v exp(x_v) / s
//   dz_v = (sum_j a_j [v = t_j] - p_v (A + b (log p_v + H))) / T        A = sum_j a_j
//
// exp and log go by powers of two: x in units of log 2.  z - m comes before the product with 1 / T: a common offset of the logits, or a mask of the type's
// lowest value in a whole row, takes nothing from x but the bits that it takes of z.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include "vectors.h"

namespace shampoo {

constexpr int LP_MAX_TOP = 64, LP_MAX_TOKENS = 64;
constexpr float LP_LN2 = 0.6931471805599453f;
constexpr float LP_NOTHING = -400.f;       // 2^x is zero from here on

// what the backward pass needs of a row
struct RowStatistics { float m, log2_s, inv_s, entropy; };

struct LogProbsArgs {
  const void *z; int64_t ld;
  const int64_t *tokens;
  float c, tau;                            // 1 / T and that over log 2
  int32_t classes, m, top;
  float *log_probs, *entropy; int64_t *top_tokens; float *top_log_probs;
  RowStatistics *stats;
  int64_t row0;
};

// Sums of a part of a row: the largest z, sum of 2^x, sum of x 2^x (x from that z, in units of log 2).  m = -infinity: nothing there.
struct SoftSums { float m, s, w; };
__device__ __forceinline__ SoftSums join_soft(const SoftSums a, const SoftSums b, float c) {
  const SoftSums hi = a.m >= b.m ? a : b, lo = a.m >= b.m ? b : a;
  if (lo.m == -INFINITY) return {hi.m, hi.s + (lo.s != lo.s ? lo.s : 0.f), hi.w};
  const float d = fmaxf((lo.m - hi.m) * c, LP_NOTHING), f = __builtin_amdgcn_exp2f(d);
  return {hi.m, fmaf(f, lo.s, hi.s), fmaf(f, fmaf(d, lo.s, lo.w), hi.w)};
}

// The order of logits: larger first, of equal ones the lower token.  0: none (masked by -infinity, or NaN).
__device__ __forceinline__ uint64_t logit_key(float z, uint32_t v) {
  if (!(z > -INFINITY)) return 0;
  const uint32_t u = __float_as_uint(z + 0.f), o = u >> 31 ? ~u : u | 0x80000000u;
  return (uint64_t)o << 32 | (0xffffffffu - v);
}
__device__ __forceinline__ float key_logit(uint64_t key) {
  const uint32_t o = (uint32_t)(key >> 32);
  return __uint_as_float(o >> 31 ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ int64_t key_token(uint64_t key) { return (int64_t)(0xffffffffu - (uint32_t)key); }

// log p of a logit from its row's statistics (a mask of the type's lowest value has one that float32 holds: no factor of 1 / log 2 on the way)
__device__ __forceinline__ float log_prob_of(float z, const RowStatistics &r, float tau) {
  if (r.m == -INFINITY) return r.log2_s != r.log2_s ? r.log2_s : -INFINITY;
  const float lp = fmaf(z - r.m, tau, -r.log2_s * LP_LN2);
  return lp > 0.f ? 0.f : lp;
}
__device__ __forceinline__ RowStatistics row_statistics(const SoftSums &t) {
  RowStatistics r;
  r.m = t.m;
  r.log2_s = t.s == 0.f ? 0.f : log2f(t.s);
  r.inv_s = t.s == 0.f ? 0.f : 1.f / t.s;                  // 0: nothing left of the row
  const float h = LP_LN2 * (r.log2_s - t.w * r.inv_s);
  r.entropy = t.s == 0.f || h < 0.f ? 0.f : h;
  return r;
}

// A workgroup per row.
template <typename T> __global__ __launch_bounds__(256) void log_probs_kernel(const LogProbsArgs g) {
  __shared__ SoftSums part[4];
  __shared__ uint64_t best[4];
  const int64_t i = g.row0 + blockIdx.x;
  const T *z = static_cast<const T *>(g.z) + i * g.ld;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  SoftSums t = {-INFINITY, 0.f, 0.f};
  for (int v = threadIdx.x; v < g.classes; v += 256) {
    const float x = load8(z, v, v + 1).v[0];
    t = join_soft(t, {x, 1.f, 0.f}, g.c);
    if (x != x) t.s = x;
    if (x == INFINITY) t.s = NAN;
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) t = join_soft(t, {__shfl_xor(t.m, o, 64), __shfl_xor(t.s, o, 64), __shfl_xor(t.w, o, 64)}, g.c);
  if (lane == 0) part[wave] = t;
  __syncthreads();
  t = part[0];
  for (int k = 1; k < 4; ++k) t = join_soft(t, part[k], g.c);
  const RowStatistics r = row_statistics(t);
  if (threadIdx.x == 0) { g.stats[i] = r; g.entropy[i] = r.entropy; }
  if ((int)threadIdx.x < g.m) {
    const int64_t tok = g.tokens[i * g.m + threadIdx.x];
    g.log_probs[i * g.m + threadIdx.x] = tok >= 0 && tok < g.classes ? log_prob_of(load8(z, (int)tok, (int)tok + 1).v[0], r, g.tau) : 0.f;
  }
  uint64_t last = ~0ull;
  for (int k = 0; k < g.top; ++k) {
    uint64_t key = 0;
    for (int v = threadIdx.x; v < g.classes; v += 256) {
      const uint64_t q = logit_key(load8(z, v, v + 1).v[0], v);
      if (q < last && q > key) key = q;
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) { const uint64_t q = __shfl_xor((unsigned long long)key, o, 64); key = q > key ? q : key; }
    __syncthreads();
    if (lane == 0) best[wave] = key;
    __syncthreads();
    for (int w = 0; w < 4; ++w) key = best[w] > key ? best[w] : key;
    if (threadIdx.x == 0) {
      g.top_tokens[i * g.top + k] = key ? key_token(key) : -1;
      g.top_log_probs[i * g.top + k] = log_prob_of(key ? key_logit(key) : -INFINITY, r, g.tau);
    }
    last = key;
  }
}

struct LogProbsGradArgs {
  const void *z; int64_t ld;
  const int64_t *tokens; const RowStatistics *stats;
  const float *a, *b;                      // gradients of the log probabilities [rows][m] and of the entropy [rows]; each may be null
  void *dz; int64_t ld_dz;                 // may be z
  float c, tau;
  int32_t classes, m;
  int64_t row0;
};
// A workgroup per row.  A token's own part is added by the thread of its first appearance, with those of all others, behind the row's other values.
template <typename T> __global__ __launch_bounds__(256) void log_probs_grad_kernel(const LogProbsGradArgs g) {
  __shared__ int32_t token[LP_MAX_TOKENS];
  __shared__ float a[LP_MAX_TOKENS];
  const int64_t i = g.row0 + blockIdx.x;
  const T *z = static_cast<const T *>(g.z) + i * g.ld;
  T *dz = static_cast<T *>(g.dz) + i * g.ld_dz;
  const RowStatistics r = g.stats[i];
  const int j = threadIdx.x;
  if (j < LP_MAX_TOKENS) {
    const int64_t t = j < g.m && g.a ? g.tokens[i * g.m + j] : -1;
    const bool valid = t >= 0 && t < g.classes;
    token[j] = valid ? (int32_t)t : -1;
    a[j] = valid ? g.a[i * g.m + j] : 0.f;
  }
  __syncthreads();
  float all = 0.f, own = 0.f;
  bool first = j < LP_MAX_TOKENS && token[j] >= 0;
  for (int k = 0; k < g.m; ++k) {
    all += a[k];
    if (first && token[k] == token[j]) { own += a[k]; if (k < j) first = false; }
  }
  const float b = g.b ? g.b[i] : 0.f, scale = -g.tau * r.inv_s;
  const bool some = r.inv_s != 0.f && (all != 0.f || b != 0.f);
  const float k1 = some ? scale * b * LP_LN2 : 0.f, k0 = some ? scale * (all + b * (r.entropy - r.log2_s * LP_LN2)) : 0.f;
  const auto value = [&](float x) {
    const float d = fmaxf((x - r.m) * g.c, LP_NOTHING);
    return some ? __builtin_amdgcn_exp2f(d) * fmaf(k1, d, k0) : 0.f;
  };
  float at_token = 0.f;
  if (first) at_token = value(load8(z, token[j], token[j] + 1).v[0]) + (r.inv_s != 0.f ? g.tau * own : 0.f);
  __syncthreads();
  for (int v = threadIdx.x * 8; v < g.classes; v += 2048) {
    f32x8 x = load8(z, v, g.classes);
#pragma unroll
    for (int e = 0; e < 8; ++e) x.v[e] = value(x.v[e]);
    store8(dz, v, g.classes, x);
  }
  __syncthreads();
  if (first) { f32x8 x = {{at_token}}; store8(dz, token[j], token[j] + 1, x); }
}

}  // namespace shampoo
