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

// Keys of which every thread of a workgroup has N (0: none; no two others alike): a bound that `top` to chosen_of(top) of them reach, or all where there are
// no more.  A search by halves below `above`, which none reaches; counts: two sets of four.
constexpr int LP_CHOSEN = 2 * LP_MAX_TOP + 16, LP_CANDIDATES = 1024;
__device__ __forceinline__ int chosen_of(int top) { return 2 * top + 16; }
__device__ __forceinline__ int count_256(int mine, int (*counts)[4], int &turn) {
  if ((threadIdx.x & 63) == 0) counts[turn][threadIdx.x >> 6] = mine;
  __syncthreads();
  const int all = counts[turn][0] + counts[turn][1] + counts[turn][2] + counts[turn][3];
  turn ^= 1;
  return all;
}
template <typename Count> __device__ __forceinline__ uint64_t bound_of(uint64_t lowest, uint64_t above, int least, int most, Count &&count) {
  if (count(lowest) <= most) return lowest;
  // from the largest on, in steps that grow: an eighth of a binade first
  uint64_t lo = lowest, hi = above, step = (uint64_t)1 << 52;
  while (hi - lo > 1) {
    const uint64_t mid = step != 0 && hi - lo > step ? hi - step : lo + (hi - lo) / 2;
    const int n = count(mid);
    if (n < least) { hi = mid; step <<= 1; }
    else if (n > most) { lo = mid; step = 0; }
    else return mid;
  }
  return lo;
}
template <int N> __device__ __forceinline__ uint64_t bound_of_keys(const uint64_t (&key)[N], uint64_t above, int top, int (*counts)[4], int &turn) {
  return bound_of(1, above, top, chosen_of(top), [&](uint64_t bound) {
    int mine = 0;
#pragma unroll
    for (int e = 0; e < N; ++e) mine += __popcll(__ballot(key[e] >= bound));
    return count_256(mine, counts, turn);
  });
}
// Candidates in LDS in their order: by how many are larger.  put(rank, key) for the first `top` of them, key 0 where there are fewer.
template <typename Put> __device__ __forceinline__ void put_in_order(const uint64_t *candidate, int n, int top, Put &&put) {
  for (int i = threadIdx.x; i < n; i += 256) {
    const uint64_t key = candidate[i];
    int rank = 0;
#pragma unroll 4
    for (int j = 0; j < n; ++j) rank += candidate[j] > key ? 1 : 0;
    if (rank < top) put(rank, key);
  }
  for (int i = n + threadIdx.x; i < top; i += 256) put(i, (uint64_t)0);
}

// A part of a row, one behind the other: `pieces` of eight logits for each thread, 2048 logits apart.
constexpr int LP_STRIPS = 4, LP_MAX_PIECES = 64, LP_MAX_PARTS = 64, LP_STEP = 2048;
constexpr float LP_SLACK = 8.f;            // x may be that far above its reference

// One workgroup per part.  One pass: sums about a reference that follows the largest at a distance, so that it hardly ever moves; and of every strip of pieces that a
// thread reads the largest logit and the first piece that has it.  The k largest strips hold the k most probable tokens (the first `top` keys of strips
// are tokens of their own, and no token of another strip comes before any of them), so that these strips alone are read again, and what reaches the bound is put in order.
// parts > 1: sums and keys of the part go to `sums` and `keys`, and log_probs_join_kernel ends the row.
struct LogPartArgs { LogProbsArgs g; int32_t parts, pieces; SoftSums *sums; uint64_t *keys; };

__device__ __forceinline__ void put_row(const LogProbsArgs &g, int64_t i, const RowStatistics &r) {
  if (threadIdx.x == 0) { g.stats[i] = r; g.entropy[i] = r.entropy; }
}
template <typename T> __device__ __forceinline__ void put_given(const LogProbsArgs &g, int64_t i, const RowStatistics &r, int j) {
  const int64_t tok = g.tokens[i * g.m + j];
  const T *z = static_cast<const T *>(g.z) + i * g.ld;
  g.log_probs[i * g.m + j] = tok >= 0 && tok < g.classes ? log_prob_of(load8(z, (int)tok, (int)tok + 1).v[0], r, g.tau) : 0.f;
}
__device__ __forceinline__ void put_top(const LogProbsArgs &g, int64_t i, const RowStatistics &r, int rank, uint64_t key) {
  g.top_tokens[i * g.top + rank] = key ? key_token(key) : -1;
  g.top_log_probs[i * g.top + rank] = log_prob_of(key ? key_logit(key) : -INFINITY, r, g.tau);
}

template <typename T, bool TOP> __global__ __launch_bounds__(256) void log_probs_kernel(const LogPartArgs a) {
  constexpr int AHEAD = 4;
  __shared__ SoftSums part_sums[4];
  const LogProbsArgs &g = a.g;
  const int64_t unit = g.row0 + blockIdx.x / (uint32_t)a.parts;
  const int part = (int)(blockIdx.x % (uint32_t)a.parts), tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const T *z = static_cast<const T *>(g.z) + unit * g.ld;
  const int begin = part * a.pieces * LP_STEP, end = min(g.classes, begin + a.pieces * LP_STEP);
  const int per_strip = (a.pieces + LP_STRIPS - 1) / LP_STRIPS;

  float ref = -INFINITY, from = 0.f, s = 0.f, w = 0.f;         // from: ref, or 0 while there is none
  float largest[LP_STRIPS];
  int at[LP_STRIPS];
#pragma unroll
  for (int k = 0; k < LP_STRIPS; ++k) { largest[k] = -INFINITY; at[k] = 0; }
  const auto take = [&](const f32x8 &x, int piece, float &top, int &top_at) {
    float m = fmaxf(fmaxf(fmaxf(x.v[0], x.v[1]), fmaxf(x.v[2], x.v[3])), fmaxf(fmaxf(x.v[4], x.v[5]), fmaxf(x.v[6], x.v[7])));
    if (m > top) { top = m; top_at = piece; }
    if (__any((m - ref) * g.c > LP_SLACK)) {
      const float next = fmaxf(ref, m);
      if (ref != -INFINITY) {
        const float d = fmaxf((ref - next) * g.c, LP_NOTHING), f = __builtin_amdgcn_exp2f(d);
        w = f * fmaf(d, s, w);
        s *= f;
      }
      ref = next;
      from = next == -INFINITY ? 0.f : next;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float d = (x.v[e] - from) * g.c, p = __builtin_amdgcn_exp2f(d);
      s += p;
      w = fmaf(p, fmaxf(d, LP_NOTHING), w);
    }
  };
#pragma unroll
  for (int k = 0; k < LP_STRIPS; ++k) {
    const int first = k * per_strip, last = min(a.pieces, first + per_strip);
    for (int q = first; q < last; q += AHEAD) {
      const int c = begin + q * LP_STEP + tid * 8;
      if (begin + q * LP_STEP >= end) break;
      Raw8<T> raw[AHEAD];
      if (q + AHEAD <= last && begin + (q + AHEAD) * LP_STEP <= end) {
#pragma unroll
        for (int e = 0; e < AHEAD; ++e) raw[e] = raw_load8(z, c + e * LP_STEP, 0x7fffffff);
#pragma unroll
        for (int e = 0; e < AHEAD; ++e) take(expand8(raw[e]), q + e, largest[k], at[k]);
      } else {
        for (int e = 0; e < AHEAD && q + e < last; ++e) {
          const int o = c + e * LP_STEP;
          if (o >= end) break;
          f32x8 x = load8(z, o, end);
#pragma unroll
          for (int v = 0; v < 8; ++v)
            if (o + v >= end) x.v[v] = -INFINITY;
          take(x, q + e, largest[k], at[k]);
        }
      }
    }
  }
  SoftSums t = {ref, s, w};
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) t = join_soft(t, {__shfl_xor(t.m, o, 64), __shfl_xor(t.s, o, 64), __shfl_xor(t.w, o, 64)}, g.c);
  if (lane == 0) part_sums[wave] = t;
  __syncthreads();
  t = part_sums[0];
#pragma unroll
  for (int k = 1; k < 4; ++k) t = join_soft(t, part_sums[k], g.c);
  const RowStatistics r = row_statistics(t);
  const int64_t out = unit * a.parts + part;
  if (a.parts == 1) {
    put_row(g, unit, r);
    if (tid < g.m) put_given<T>(g, unit, r, tid);
  } else if (tid == 0) a.sums[out] = t;

  if constexpr (TOP) {
    __shared__ int counts[2][4], chosen[LP_CHOSEN], n_chosen, n_candidates;
    __shared__ uint64_t candidate[LP_CANDIDATES];
    int turn = 0;
    uint64_t key[LP_STRIPS];
    float most = -INFINITY;
#pragma unroll
    for (int k = 0; k < LP_STRIPS; ++k) { key[k] = logit_key(largest[k], begin + at[k] * LP_STEP + tid * 8); most = fmaxf(most, largest[k]); }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) most = fmaxf(most, __shfl_xor(most, o, 64));
    __syncthreads();                       // part_sums have been read
    if (lane == 0) part_sums[wave].m = most;
    if (tid == 0) n_chosen = n_candidates = 0;
    __syncthreads();
    most = fmaxf(fmaxf(part_sums[0].m, part_sums[1].m), fmaxf(part_sums[2].m, part_sums[3].m));
    const uint64_t above = logit_key(most, 0) + 1;
    uint64_t bound = bound_of_keys(key, above, g.top, counts, turn);
#pragma unroll
    for (int k = 0; k < LP_STRIPS; ++k)
      if (key[k] >= bound) { const int n = atomicAdd(&n_chosen, 1); if (n < LP_CHOSEN) chosen[n] = k * 256 + tid; }
    __syncthreads();
    const int strips = min(n_chosen, LP_CHOSEN), again = strips * per_strip;
    // the chosen strips' logits
    const auto each = [&](auto &&f) {
      for (int i = tid; i < again; i += 256) {
        const int u = i / strips, strip = chosen[i - u * strips], q = (strip >> 8) * per_strip + u, o = begin + q * LP_STEP + (strip & 255) * 8;
        if (q >= min(a.pieces, ((strip >> 8) + 1) * per_strip) || o >= end) continue;
        const f32x8 x = load8(z, o, end);
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (o + e < end) f(logit_key(x.v[e], o + e));
      }
    };
    // a bound that is a strip's counts its whole piece: its other tokens may come before the next strip's
    each([&](uint64_t k) {
      if (k && (k | 7) >= bound) { const int n = atomicAdd(&n_candidates, 1); if (n < LP_CANDIDATES) candidate[n] = k; }
    });
    __syncthreads();
    if (n_candidates > LP_CANDIDATES) {    // many tokens of one strip: a bound among the tokens themselves
      bound = bound_of(max(bound & ~(uint64_t)7, (uint64_t)1), above, g.top, LP_CANDIDATES, [&](uint64_t b) {
        int mine = 0;
        each([&](uint64_t k) { mine += k >= b ? 1 : 0; });
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) mine += __shfl_xor(mine, o, 64);
        return count_256(mine, counts, turn);
      });
      __syncthreads();
      if (tid == 0) n_candidates = 0;
      __syncthreads();
      each([&](uint64_t k) {
        if (k >= bound) { const int n = atomicAdd(&n_candidates, 1); if (n < LP_CANDIDATES) candidate[n] = k; }
      });
      __syncthreads();
    }
    put_in_order(candidate, min(n_candidates, LP_CANDIDATES), g.top, [&](int rank, uint64_t k) {
      if (a.parts == 1) put_top(g, unit, r, rank, k); else a.keys[out * g.top + rank] = k;
    });
  }
}

// The parts of a row together: sums in order, and of the keys those that reach a bound.
template <typename T> __global__ __launch_bounds__(256) void log_probs_join_kernel(const LogPartArgs a) {
  constexpr int N = LP_MAX_PARTS * LP_MAX_TOP / 256;
  __shared__ int counts[2][4], n_candidates;
  __shared__ uint64_t candidate[LP_CHOSEN];
  const LogProbsArgs &g = a.g;
  const int64_t i = g.row0 + blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63;
  SoftSums t = {-INFINITY, 0.f, 0.f};
  if (lane < a.parts) t = a.sums[i * a.parts + lane];
  uint64_t key[N];
  const int n = a.parts * g.top;
#pragma unroll
  for (int e = 0; e < N; ++e) key[e] = e * 256 + tid < n ? a.keys[i * n + e * 256 + tid] : 0;
  if (tid == 0) n_candidates = 0;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) t = join_soft(t, {__shfl_xor(t.m, o, 64), __shfl_xor(t.s, o, 64), __shfl_xor(t.w, o, 64)}, g.c);
  const RowStatistics r = row_statistics(t);
  put_row(g, i, r);
  if (tid < g.m) put_given<T>(g, i, r, tid);
  if (g.top == 0) return;
  __shared__ uint64_t part_most[4];
  uint64_t most = 0;
#pragma unroll
  for (int e = 0; e < N; ++e) most = max(most, key[e]);
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) most = max(most, (uint64_t)__shfl_xor((unsigned long long)most, o, 64));
  if (lane == 0) part_most[tid >> 6] = most;
  __syncthreads();
  most = max(max(part_most[0], part_most[1]), max(part_most[2], part_most[3]));
  int turn = 0;
  const uint64_t bound = bound_of_keys(key, most + 1, g.top, counts, turn);
#pragma unroll
  for (int e = 0; e < N; ++e)
    if (key[e] >= bound) { const int k = atomicAdd(&n_candidates, 1); if (k < LP_CHOSEN) candidate[k] = key[e]; }
  __syncthreads();
  put_in_order(candidate, min(n_candidates, LP_CHOSEN), g.top, [&](int rank, uint64_t k) { put_top(g, i, r, rank, k); });
}

struct LogProbsGradArgs {
  const void *z; int64_t ld;
  const int64_t *tokens; const RowStatistics *stats;
  const float *a, *b;                      // gradients of the log probabilities [rows][m] and of the entropy [rows]; each may be null
  void *dz; int64_t ld_dz;                 // may be z
  float c, tau;
  int32_t classes, m, parts, part_len;     // part_len: classes of a part, a multiple of LP_STEP
  int64_t row0;
};
// A workgroup per part of a row.  A token's own part is added by the thread of its first appearance, with those of all others, behind the row's other values.
template <typename T> __global__ __launch_bounds__(256) void log_probs_grad_kernel(const LogProbsGradArgs g) {
  __shared__ int32_t token[LP_MAX_TOKENS];
  __shared__ float a[LP_MAX_TOKENS];
  const int64_t i = g.row0 + blockIdx.x / (uint32_t)g.parts;
  const int begin = (int)(blockIdx.x % (uint32_t)g.parts) * g.part_len, end = min(g.classes, begin + g.part_len);
  const T *z = static_cast<const T *>(g.z) + i * g.ld;
  T *dz = static_cast<T *>(g.dz) + i * g.ld_dz;
  if (begin >= end) return;
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
  bool first = j < LP_MAX_TOKENS && token[j] >= begin && token[j] < end;
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
  for (int v = begin + threadIdx.x * 8; v < end; v += LP_STEP) {
    f32x8 x = load8(z, v, g.classes);
#pragma unroll
    for (int e = 0; e < 8; ++e) x.v[e] = value(x.v[e]);
    store8(dz, v, g.classes, x);
  }
  __syncthreads();
  if (first) { f32x8 x = {{at_token}}; store8(dz, token[j], token[j] + 1, x); }
}

}  // namespace shampoo
