// Residual sum with the norms after and before a block, its gate and its scale:
//
//   u = norm_post(f)        r' = r + alpha gate u        h = norm_pre(r')
//   norm(x) = (x - mean) / sqrt(mean of squares of that + eps) w + b     (RMS: without mean and b)
//
// and its gradients, from r and f as they were or as 8-bit checkpoints (checkpoint.h) hold them:
//
//   dr = dr' + inv (g - n mean(g n) - mean(g)),  g = dh w_pre, n the normalised r'  (RMS: without mean(g))
//   du = alpha gate dr,  df the same of norm_post,  dgate = sum alpha u dr,  dw = sum dy n,  db = sum dy
//
// A team of threads holds a row in registers, in pieces of eight neighbouring features per thread, so that memory is read and
// written once: bound by memory, beside about 35 vector operations per element.  Forward a team is one wavefront up to
// 2048 features: its sums need no barrier, and other wavefronts hide its latency.  Backward a team has several rows, the next one on its way
// while one is worked on, and keeps weights and the sums for their gradients in registers, so a thread has one piece
// (up to 4096 features): 16384 x 2048 in bf16 from checkpoints 84 us, where a wavefront per row with four pieces a thread (477 registers) took 223 and
// weights read for every row 141; 768 teams of 256 threads, three per CU (with 1024 teams a fifth more).  The teams' sums are joined in order by a second launch.
// 16384 x 2048, bf16: forward with checkpoints 72 us (337 MB, 4.7 TB/s), backward 84 + 7 us (337 MB, 3.7 TB/s: 57 vector
// operations per element beside them).  3003 x 1001, float32, layer norms: 14 and 22 + 6 us.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include "checkpoint.h"
#include "vectors.h"

namespace shampoo {

enum { NORM_NONE = 0, NORM_RMS = 1, NORM_LAYER = 2 };

struct ResidualNormArgs {
  const void *r, *f; int64_t ldr, ldf;                 // rows as they were, or
  Packed r8, f8;                                       // their checkpoints (forward: written where codes are given)
  const float *w_post, *b_post, *gate, *w_pre, *b_pre; // [cols], gate [groups][cols]
  void *r_out, *h; int64_t ld_r_out, ldh;              // forward
  const void *dr_out, *dh; int64_t ld_dr_out, ld_dh;   // backward
  void *dr, *df; int64_t ld_dr, ld_df;
  float *dgate;                                        // written here where a team has whole groups
  float *partial;                                      // [teams][5][cols]: dgate, dw_post, dw_pre, db_post, db_pre
  int64_t rows, group_rows, chunk_rows, teams;         // rows per gate, per team of the backward pass
  int64_t row0;                                        // forward: this launch's first row
  int32_t chunks_per_group;                            // 0: a team has whole groups
  int32_t cols, post, pre;
  float epsilon, alpha;
};
enum { SUM_GATE = 0, SUM_W_POST = 1, SUM_W_PRE = 2, SUM_B_POST = 3, SUM_B_PRE = 4, SUMS = 5 };

// The sum over a wavefront, in every lane: within rows of 16 lanes, then across them.
__device__ __forceinline__ float wave_sum(float x) {
#define ADD_DPP(CTRL, ROWS) x += __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(x), CTRL, ROWS, 0xf, false))
  ADD_DPP(0x111, 0xf); ADD_DPP(0x112, 0xf); ADD_DPP(0x114, 0xf); ADD_DPP(0x118, 0xf);      // row_shr 1, 2, 4, 8
  ADD_DPP(0x142, 0xa); ADD_DPP(0x143, 0xc);                                                // row_bcast 15, 31
#undef ADD_DPP
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), 63));
}
// sums over the threads of a row, for all of them; `slot` (two floats per wavefront): one that no other sum uses at the time.  BOTH:
// of x and y, otherwise of x alone.
template <int TPR, bool BOTH> __device__ __forceinline__ void row_sums(float &x, float &y, float *slot) {
  x = wave_sum(x);
  if constexpr (BOTH) y = wave_sum(y);
  if constexpr (TPR > 64) {
    constexpr int WAVES = TPR / 64;
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) { slot[wave] = x; if constexpr (BOTH) slot[WAVES + wave] = y; }
    __syncthreads();
    auto all = [](const float *p) {
      float s = p[0] + p[1];
      if constexpr (WAVES >= 4) s += p[2] + p[3];
      if constexpr (WAVES == 8) s += (p[4] + p[5]) + (p[6] + p[7]);
      return s;
    };
    x = all(slot);
    if constexpr (BOTH) y = all(slot + WAVES);
  }
}
constexpr int NORM_SLOT = 16;       // floats of a slot

// Where a thread's pieces of a row are: piece j at column (at + TPR j) 8.
template <int TPR, int NJ> struct RowPieces {
  int at, cols;
  __device__ __forceinline__ int column(int j) const { return (at + TPR * j) * 8; }
  __device__ __forceinline__ bool has(int j, int e) const { return column(j) + e < cols; }
};

// x becomes (x - mean) / sqrt(...), the returned value one over the root.  Padding stays zero.  Uses slots 0 and 1.
template <int TPR, int NJ> __device__ __forceinline__ float normalise(f32x8 (&x)[NJ], const RowPieces<TPR, NJ> &at, int kind, float eps, float *slot) {
  const float per = 1.f / (float)at.cols;
  float s = 0.f, unused = 0.f;
  if (kind == NORM_LAYER) {
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) s += x[j].v[e];
    row_sums<TPR, false>(s, unused, slot);
    const float mean = s * per;
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) x[j].v[e] = at.has(j, e) ? x[j].v[e] - mean : 0.f;
    s = 0.f;
  }
#pragma unroll
  for (int j = 0; j < NJ; ++j)
#pragma unroll
    for (int e = 0; e < 8; ++e) s += x[j].v[e] * x[j].v[e];
  row_sums<TPR, false>(s, unused, slot + NORM_SLOT);
  const float inv = rsqrtf(s * per + eps);
#pragma unroll
  for (int j = 0; j < NJ; ++j)
#pragma unroll
    for (int e = 0; e < 8; ++e) x[j].v[e] *= inv;
  return inv;
}

template <typename T, int TPR, int NJ>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void residual_norm_forward_kernel(const ResidualNormArgs g) {
  constexpr int TEAMS = TPR > 256 ? 1 : 256 / TPR;
  __shared__ float red[4 * NORM_SLOT];
  const RowPieces<TPR, NJ> at = {(int)threadIdx.x % TPR, g.cols};
  const int64_t i = g.row0 + (int64_t)blockIdx.x * TEAMS + threadIdx.x / TPR;
  if (i >= g.rows) return;                             // a whole team
  f32x8 f[NJ], r[NJ];
  const T *pr = static_cast<const T *>(g.r) + i * g.ldr, *pf = static_cast<const T *>(g.f) + i * g.ldf;
#pragma unroll
  for (int j = 0; j < NJ; ++j) f[j] = load8(pf, at.column(j), g.cols);
#pragma unroll
  for (int j = 0; j < NJ; ++j) r[j] = load8(pr, at.column(j), g.cols);
  if (g.f8.codes) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) { packed_store8(g.f8, i, at.column(j), f[j]); packed_store8(g.r8, i, at.column(j), r[j]); }
  }
  if (g.post != NORM_NONE) {
    normalise(f, at, g.post, g.epsilon, red);
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const f32x8 w = load8(g.w_post, at.column(j), g.cols);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[j].v[e] *= w.v[e];
    }
    if (g.b_post) {
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const f32x8 b = load8(g.b_post, at.column(j), g.cols);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[j].v[e] += b.v[e];
      }
    }
  }
  if (g.gate) {
    const float *gate = g.gate + i / g.group_rows * g.cols;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const f32x8 w = load8(gate, at.column(j), g.cols);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[j].v[e] *= w.v[e];
    }
  }
  T *po = static_cast<T *>(g.r_out) + i * g.ld_r_out;
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
#pragma unroll
    for (int e = 0; e < 8; ++e) r[j].v[e] += g.alpha * f[j].v[e];
    store8(po, at.column(j), g.cols, r[j]);
  }
  if (g.pre == NORM_NONE) return;
  normalise(r, at, g.pre, g.epsilon, red + 2 * NORM_SLOT);
  T *ph = static_cast<T *>(g.h) + i * g.ldh;
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    const f32x8 w = load8(g.w_pre, at.column(j), g.cols);
    f32x8 b = {{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}};
    if (g.b_pre) b = load8(g.b_pre, at.column(j), g.cols);
#pragma unroll
    for (int e = 0; e < 8; ++e) r[j].v[e] = r[j].v[e] * w.v[e] + b.v[e];
    store8(ph, at.column(j), g.cols, r[j]);
  }
}

// dx of a norm in place of dy w (in `d`): inv (d - n mean(d n) - mean(d)).  Padding stays zero.
template <int TPR, int NJ> __device__ __forceinline__ void norm_gradient(f32x8 (&d)[NJ], const f32x8 (&n)[NJ], const RowPieces<TPR, NJ> &at, float inv, int kind, float *slot) {
  float sn = 0.f, s = 0.f;
#pragma unroll
  for (int j = 0; j < NJ; ++j)
#pragma unroll
    for (int e = 0; e < 8; ++e) sn += d[j].v[e] * n[j].v[e];
  const float per = -inv / (float)at.cols;
  if (kind == NORM_LAYER) {
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) s += d[j].v[e];
    row_sums<TPR, true>(sn, s, slot);
    sn *= per; s *= per;
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) d[j].v[e] = at.has(j, e) ? inv * d[j].v[e] + (n[j].v[e] * sn + s) : 0.f;
  } else {
    row_sums<TPR, false>(sn, s, slot);
    sn *= per;
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) d[j].v[e] = inv * d[j].v[e] + n[j].v[e] * sn;
  }
}

// What a row brings, as it comes from memory: r and f as eight values, or eight codes and their exponent byte in the same registers.
template <typename T, int NJ> struct RawRow {
  Raw8<T> r[NJ], f[NJ], dr_out[NJ], dh[NJ];
  uint32_t r_byte[NJ], f_byte[NJ];
  template <typename At> __device__ __forceinline__ void load(const ResidualNormArgs &g, const At &at, int64_t i) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int c = at.column(j);
      if (g.r8.codes) { codes(g.f8, i, c, f[j], f_byte[j]); codes(g.r8, i, c, r[j], r_byte[j]); }
      else {
        f[j] = raw_load8(static_cast<const T *>(g.f) + i * g.ldf, c, g.cols);
        r[j] = raw_load8(static_cast<const T *>(g.r) + i * g.ldr, c, g.cols);
      }
      if (g.dh) dh[j] = raw_load8(static_cast<const T *>(g.dh) + i * g.ld_dh, c, g.cols);
      if (g.dr_out) dr_out[j] = raw_load8(static_cast<const T *>(g.dr_out) + i * g.ld_dr_out, c, g.cols);
    }
  }
  __device__ __forceinline__ void codes(const Packed &p, int64_t i, int c, Raw8<T> &x, uint32_t &byte) {
    uint2 w = make_uint2(0u, 0u);
    byte = 0u;
    if (c < p.cols) {
      w = *reinterpret_cast<const uint2 *>(p.codes + i * p.pitch + c);
      byte = p.exps[i * (p.pitch >> 5) + (c >> 5)];
    }
    x.u[0][0] = w.x; x.u[0][1] = w.y;
  }
  // a group that is not finite reads NaN in the padding too
  template <typename At> static __device__ __forceinline__ f32x8 values(const Raw8<T> &x, uint32_t byte, bool packed, const At &at, int j) {
    if (!packed) return expand8(x);
    f32x8 v = unpack8(make_uint2(x.u[0][0], x.u[0][1]), value_per_code(byte));
    if (at.column(j) + 8 > at.cols) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v.v[e] = at.has(j, e) ? v.v[e] : 0.f;
    }
    return v;
  }
};

// Rows of weights (times alpha), kept in registers over a team's rows where a thread has one piece, and otherwise read where they
// are used.  No weights: ones.
template <int NJ> struct NormWeight {
  static constexpr bool KEEP = NJ == 1;
  f32x8 kept;
  const float *p;
  float alpha;
  template <typename At> __device__ __forceinline__ void set(const float *w, const At &at, float by = 1.f) {
    p = w; alpha = by;
    if constexpr (KEEP) kept = read(at, 0);
  }
  template <typename At> __device__ __forceinline__ f32x8 read(const At &at, int j) const {
    f32x8 x = {{alpha, alpha, alpha, alpha, alpha, alpha, alpha, alpha}};
    if (p) {
      x = load8(p, at.column(j), at.cols);
#pragma unroll
      for (int e = 0; e < 8; ++e) x.v[e] *= alpha;
    }
    return x;
  }
  template <typename At> __device__ __forceinline__ f32x8 get(const At &at, int j) const {
    if constexpr (KEEP) return kept; else return read(at, j);
  }
};

// A team has chunk_rows rows of one group, or of whole groups, and their sums for the weights.  BIAS: of biases too.
template <typename T, int TPR, int NJ, bool BIAS>
__global__ __launch_bounds__(TPR == 64 ? 256 : TPR, NJ == 1 && TPR <= 256 && sizeof(T) == 2 && !BIAS ? 3 : 1) void residual_norm_backward_kernel(const ResidualNormArgs g) {
  constexpr int TEAMS = TPR == 64 ? 4 : 1, NSUM = BIAS ? 5 : 3;
  __shared__ float red[2][6 * NORM_SLOT];
  const RowPieces<TPR, NJ> at = {(int)threadIdx.x % TPR, g.cols};
  const int64_t team = (int64_t)blockIdx.x * TEAMS + threadIdx.x / TPR;
  if (team >= g.teams) return;
  int64_t i0, i1;
  if (g.chunks_per_group) {
    const int64_t group = team / g.chunks_per_group, k = team - group * g.chunks_per_group;
    i0 = group * g.group_rows + k * g.chunk_rows;
    i1 = min(i0 + g.chunk_rows, (group + 1) * g.group_rows);
  } else {
    i0 = team * g.chunk_rows;
    i1 = min(i0 + g.chunk_rows, g.rows);
  }
  f32x8 sum[NSUM][NJ];
#pragma unroll
  for (int q = 0; q < NSUM; ++q)
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[q][j].v[e] = 0.f;
  int64_t left = g.chunks_per_group ? 0 : g.group_rows, group = g.gate ? i0 / g.group_rows : 0;   // rows until the group's sum is written
  NormWeight<NJ> w_post, b_post, w_pre, gate;
  w_post.set(g.post != NORM_NONE ? g.w_post : nullptr, at); w_pre.set(g.pre != NORM_NONE ? g.w_pre : nullptr, at);
  b_post.set(BIAS ? g.b_post : nullptr, at);
  gate.set(g.gate ? g.gate + group * g.cols : nullptr, at, g.alpha);
  RawRow<T, NJ> raw;
  if (i0 < i1) raw.load(g, at, i0);
  for (int64_t i = i0; i < i1; ++i) {
    float *slot = red[i & 1];
    f32x8 r[NJ], f[NJ], d[NJ];
    Raw8<T> over[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      f[j] = raw.values(raw.f[j], raw.f_byte[j], g.r8.codes != nullptr, at, j);
      r[j] = raw.values(raw.r[j], raw.r_byte[j], g.r8.codes != nullptr, at, j);
      if (g.dh) d[j] = expand8(raw.dh[j]);
      over[j] = raw.dr_out[j];
    }
    if (i + 1 < i1) raw.load(g, at, i + 1);
    const float inv_f = g.post != NORM_NONE ? normalise(f, at, g.post, g.epsilon, slot) : 1.f;
    // u = norm_post(f), formed again where it is needed
    auto block = [&](int j) {
      f32x8 u = f[j];
      if (g.post != NORM_NONE) {
        const f32x8 w = w_post.get(at, j);
#pragma unroll
        for (int e = 0; e < 8; ++e) u.v[e] *= w.v[e];
        if (BIAS && g.b_post) {
          const f32x8 b = b_post.get(at, j);
#pragma unroll
          for (int e = 0; e < 8; ++e) u.v[e] += b.v[e];
        }
      }
      return u;
    };
    if (g.pre != NORM_NONE) {
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const f32x8 u = block(j), w = gate.get(at, j);
#pragma unroll
        for (int e = 0; e < 8; ++e) r[j].v[e] += w.v[e] * u.v[e];
      }
      const float inv = normalise(r, at, g.pre, g.epsilon, slot + 2 * NORM_SLOT);
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const f32x8 w = w_pre.get(at, j);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          sum[SUM_W_PRE][j].v[e] += d[j].v[e] * r[j].v[e];
          if constexpr (BIAS) sum[SUM_B_PRE][j].v[e] += d[j].v[e];
          d[j].v[e] *= w.v[e];
        }
      }
      norm_gradient<TPR, NJ>(d, r, at, inv, g.pre, slot + 4 * NORM_SLOT);
    } else {
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) d[j].v[e] = 0.f;
    }
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      if (g.dr_out) {
        const f32x8 x = expand8(over[j]);
#pragma unroll
        for (int e = 0; e < 8; ++e) d[j].v[e] += x.v[e];
      }
      store8(static_cast<T *>(g.dr) + i * g.ld_dr, at.column(j), g.cols, d[j]);
      if (g.gate) {                                     // times alpha at the end
        const f32x8 u = block(j);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[SUM_GATE][j].v[e] += d[j].v[e] * u.v[e];
      }
      const f32x8 w = gate.get(at, j);
#pragma unroll
      for (int e = 0; e < 8; ++e) d[j].v[e] *= w.v[e];
      if (g.post != NORM_NONE) {
        const f32x8 w = w_post.get(at, j);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          sum[SUM_W_POST][j].v[e] += d[j].v[e] * f[j].v[e];
          if constexpr (BIAS) sum[SUM_B_POST][j].v[e] += d[j].v[e];
          d[j].v[e] *= w.v[e];
        }
      }
    }
    if (g.post != NORM_NONE) norm_gradient<TPR, NJ>(d, f, at, inv_f, g.post, slot + 5 * NORM_SLOT);
#pragma unroll
    for (int j = 0; j < NJ; ++j) store8(static_cast<T *>(g.df) + i * g.ld_df, at.column(j), g.cols, d[j]);
    if (left && --left == 0) {
      if (g.dgate) {
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
#pragma unroll
          for (int e = 0; e < 8; ++e) sum[SUM_GATE][j].v[e] *= g.alpha;
          store8(g.dgate + group * g.cols, at.column(j), g.cols, sum[SUM_GATE][j]);
        }
      }
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[SUM_GATE][j].v[e] = 0.f;
      left = g.group_rows;
      ++group;
      if (g.gate && i + 1 < i1) gate.set(g.gate + group * g.cols, at, g.alpha);
    }
  }
  float *out = g.partial + team * SUMS * g.cols;
#pragma unroll
  for (int q = 0; q < NSUM; ++q) {
    const bool wanted = q == SUM_GATE ? g.gate && g.chunks_per_group : q == SUM_W_POST ? g.post != NORM_NONE : q == SUM_W_PRE ? g.pre != NORM_NONE : true;
    if (!wanted) continue;
    if (q == SUM_GATE) {
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[SUM_GATE][j].v[e] *= g.alpha;
    }
#pragma unroll
    for (int j = 0; j < NJ; ++j) store8(out + q * g.cols, at.column(j), g.cols, sum[q][j]);
  }
}

// Sums over teams or parts: out_k[o][j] = (add: out_k[o][j] +) sum over p < parts_k of in_k[o][p][j], k = blockIdx.z, o = blockIdx.y, in an order that
// does not depend on the launch.  A workgroup has 64 columns and 16 threads for each.
constexpr int JOIN_SUMS = 8;
struct JoinSumsArgs {
  const float *in[JOIN_SUMS]; float *out[JOIN_SUMS]; int32_t parts[JOIN_SUMS];
  int64_t output_stride, part_stride, out_stride;
  int32_t cols, add;
};
__global__ __launch_bounds__(1024) void join_sums_kernel(const JoinSumsArgs g) {
  __shared__ float part[16][64];
  const int c = threadIdx.x & 63, k = threadIdx.x >> 6, j = blockIdx.x * 64 + c, parts = g.parts[blockIdx.z];
  float s[4] = {0.f, 0.f, 0.f, 0.f};
  if (j < g.cols) {
    const float *p = g.in[blockIdx.z] + blockIdx.y * g.output_stride + j;
    int i = k;
    for (; i + 240 < parts; i += 256) {
      float x[16];
#pragma unroll
      for (int q = 0; q < 16; ++q) x[q] = p[(i + 16 * q) * g.part_stride];
#pragma unroll
      for (int q = 0; q < 16; ++q) s[q & 3] += x[q];
    }
    for (; i + 48 < parts; i += 64) {
#pragma unroll
      for (int q = 0; q < 4; ++q) s[q] += p[(i + 16 * q) * g.part_stride];
    }
    for (; i < parts; i += 16) s[0] += p[i * g.part_stride];
  }
  part[k][c] = (s[0] + s[1]) + (s[2] + s[3]);
  __syncthreads();
  if (k != 0 || j >= g.cols) return;
  float t = 0.f;
#pragma unroll
  for (int q = 0; q < 16; ++q) t += part[q][c];
  float *out = g.out[blockIdx.z] + blockIdx.y * g.out_stride + j;
  *out = g.add ? *out + t : t;
}

}  // namespace shampoo
