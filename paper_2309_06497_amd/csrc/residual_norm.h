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
// A row is held in registers, in pieces of eight neighbouring features per thread, so that memory is read and written once.
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
  float *dgate;                                        // written here where a workgroup has whole groups
  float *partial;                                      // [workgroups][5][cols]: dgate, dw_post, db_post, dw_pre, db_pre
  int64_t rows, group_rows, chunk_rows;                // rows per gate, per workgroup
  int32_t chunks_per_group;                            // 0: a workgroup has whole groups
  int32_t cols, post, pre;
  float epsilon, alpha;
  int32_t vec;                                         // rows start on multiples of 16 bytes
};

// sums over the threads of a row, for all of them; `slot` (two floats per wavefront): one that no other sum uses at the time
template <int TPR> __device__ __forceinline__ void row_sums(float &x, float &y, float *slot) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) { x += __shfl_xor(x, o, 64); y += __shfl_xor(y, o, 64); }
  if constexpr (TPR == 256) {
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) { slot[2 * wave] = x; slot[2 * wave + 1] = y; }
    __syncthreads();
    x = (slot[0] + slot[2]) + (slot[4] + slot[6]);
    y = (slot[1] + slot[3]) + (slot[5] + slot[7]);
  }
}

// x becomes (x - mean) / sqrt(...), the returned value one over the root.  Padding stays zero.
template <int TPR, int NJ> __device__ __forceinline__ float normalise(f32x8 (&x)[NJ], int kind, int cols, float eps, int at, float *slot) {
  const float per = 1.f / (float)cols;
  float s = 0.f, unused = 0.f;
  if (kind == NORM_LAYER) {
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) s += x[j].v[e];
    row_sums<TPR>(s, unused, slot);
    const float mean = s * per;
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) x[j].v[e] = (at + TPR * j) * 8 + e < cols ? x[j].v[e] - mean : 0.f;
    s = 0.f;
  }
#pragma unroll
  for (int j = 0; j < NJ; ++j)
#pragma unroll
    for (int e = 0; e < 8; ++e) s += x[j].v[e] * x[j].v[e];
  row_sums<TPR>(s, unused, slot + 8);
  const float inv = rsqrtf(s * per + eps);
#pragma unroll
  for (int j = 0; j < NJ; ++j)
#pragma unroll
    for (int e = 0; e < 8; ++e) x[j].v[e] *= inv;
  return inv;
}

template <typename T, int TPR, int NJ> __global__ __launch_bounds__(256) void residual_norm_forward_kernel(const ResidualNormArgs g) {
  __shared__ float red[32];
  const int at = threadIdx.x % TPR;
  const int64_t i = (int64_t)blockIdx.x * (256 / TPR) + threadIdx.x / TPR;
  if (i >= g.rows) return;                             // a whole wavefront; workgroups of one row have one
  f32x8 f[NJ], r[NJ];
  const T *pr = static_cast<const T *>(g.r) + i * g.ldr, *pf = static_cast<const T *>(g.f) + i * g.ldf;
#pragma unroll
  for (int j = 0; j < NJ; ++j) f[j] = load8(pf, (at + TPR * j) * 8, g.cols, g.vec);
#pragma unroll
  for (int j = 0; j < NJ; ++j) r[j] = load8(pr, (at + TPR * j) * 8, g.cols, g.vec);
  if (g.f8.codes) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) { packed_store8(g.f8, i, (at + TPR * j) * 8, f[j]); packed_store8(g.r8, i, (at + TPR * j) * 8, r[j]); }
  }
  if (g.post != NORM_NONE) normalise<TPR, NJ>(f, g.post, g.cols, g.epsilon, at, red);
  const float *gate = g.gate ? g.gate + i / g.group_rows * g.cols : nullptr;
  T *po = static_cast<T *>(g.r_out) + i * g.ld_r_out;
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    const int c = (at + TPR * j) * 8;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (c + e >= g.cols) continue;
      float u = f[j].v[e];
      if (g.post != NORM_NONE) { u *= g.w_post[c + e]; if (g.b_post) u += g.b_post[c + e]; }
      if (gate) u *= gate[c + e];
      r[j].v[e] += g.alpha * u;
    }
    store8(po, c, g.cols, g.vec, r[j]);
  }
  if (g.pre == NORM_NONE) return;
  normalise<TPR, NJ>(r, g.pre, g.cols, g.epsilon, at, red + 16);
  T *ph = static_cast<T *>(g.h) + i * g.ldh;
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    const int c = (at + TPR * j) * 8;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (c + e >= g.cols) continue;
      r[j].v[e] *= g.w_pre[c + e];
      if (g.b_pre) r[j].v[e] += g.b_pre[c + e];
    }
    store8(ph, c, g.cols, g.vec, r[j]);
  }
}

// dx of a norm in place of dy w (in `d`): inv (d - n mean(d n) - mean(d))
template <int NJ> __device__ __forceinline__ void norm_gradient(f32x8 (&d)[NJ], const f32x8 (&n)[NJ], float inv, int kind, int cols, float *slot) {
  float sn = 0.f, s = 0.f;
#pragma unroll
  for (int j = 0; j < NJ; ++j)
#pragma unroll
    for (int e = 0; e < 8; ++e) { sn += d[j].v[e] * n[j].v[e]; s += d[j].v[e]; }
  row_sums<256>(sn, s, slot);
  const float per = 1.f / (float)cols;
  sn *= per; s = kind == NORM_LAYER ? s * per : 0.f;
#pragma unroll
  for (int j = 0; j < NJ; ++j)
#pragma unroll
    for (int e = 0; e < 8; ++e) d[j].v[e] = inv * (d[j].v[e] - n[j].v[e] * sn - s);
}

// A workgroup has chunk_rows rows of one group, or of whole groups, and their sums for the weights.
template <typename T, bool PACKED, int NJ> __global__ __launch_bounds__(256) void residual_norm_backward_kernel(const ResidualNormArgs g) {
  __shared__ float red[2][56];
  const int at = threadIdx.x;
  int64_t i0, i1;
  if (g.chunks_per_group) {
    const int64_t group = blockIdx.x / g.chunks_per_group, k = blockIdx.x - group * g.chunks_per_group;
    i0 = group * g.group_rows + k * g.chunk_rows;
    i1 = min(i0 + g.chunk_rows, (group + 1) * g.group_rows);
  } else {
    i0 = (int64_t)blockIdx.x * g.chunk_rows;
    i1 = min(i0 + g.chunk_rows, g.rows);
  }
  f32x8 sum[5][NJ];
#pragma unroll
  for (int q = 0; q < 5; ++q)
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[q][j].v[e] = 0.f;
  int64_t left = g.chunks_per_group ? 0 : g.group_rows, group = g.gate ? i0 / g.group_rows : 0;   // rows until the group's sum is written
  for (int64_t i = i0; i < i1; ++i) {
    float *slot = red[i & 1];
    f32x8 r[NJ], f[NJ], u[NJ], d[NJ];
    const float *gate = g.gate ? g.gate + group * g.cols : nullptr;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int c = (at + 256 * j) * 8;
      if constexpr (PACKED) {
        f32x8 zero = {{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}};
        f[j] = c < g.cols ? packed_load8(g.f8, i, c) : zero;
        r[j] = c < g.cols ? packed_load8(g.r8, i, c) : zero;
        // a group that is not finite reads NaN in the padding too
#pragma unroll
        for (int e = 0; e < 8; ++e) if (c + e >= g.cols) { f[j].v[e] = 0.f; r[j].v[e] = 0.f; }
      } else {
        f[j] = load8(static_cast<const T *>(g.f) + i * g.ldf, c, g.cols, g.vec);
        r[j] = load8(static_cast<const T *>(g.r) + i * g.ldr, c, g.cols, g.vec);
      }
    }
    const float inv_f = g.post != NORM_NONE ? normalise<256, NJ>(f, g.post, g.cols, g.epsilon, at, slot) : 1.f;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int c = (at + 256 * j) * 8;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        u[j].v[e] = f[j].v[e];
        if (c + e >= g.cols) continue;
        if (g.post != NORM_NONE) { u[j].v[e] *= g.w_post[c + e]; if (g.b_post) u[j].v[e] += g.b_post[c + e]; }
        r[j].v[e] += g.alpha * (gate ? gate[c + e] * u[j].v[e] : u[j].v[e]);
      }
    }
    if (g.pre != NORM_NONE) {
      const float inv = normalise<256, NJ>(r, g.pre, g.cols, g.epsilon, at, slot + 16);
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const int c = (at + 256 * j) * 8;
        d[j] = load8(static_cast<const T *>(g.dh) + i * g.ld_dh, c, g.cols, g.vec);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          sum[3][j].v[e] += d[j].v[e] * r[j].v[e];
          sum[4][j].v[e] += d[j].v[e];
          d[j].v[e] *= c + e < g.cols ? g.w_pre[c + e] : 0.f;
        }
      }
      norm_gradient<NJ>(d, r, inv, g.pre, g.cols, slot + 32);
    } else {
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) d[j].v[e] = 0.f;
    }
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int c = (at + 256 * j) * 8;
      if (g.dr_out) {
        const f32x8 x = load8(static_cast<const T *>(g.dr_out) + i * g.ld_dr_out, c, g.cols, g.vec);
#pragma unroll
        for (int e = 0; e < 8; ++e) d[j].v[e] += x.v[e];
      }
      if (g.dr) store8(static_cast<T *>(g.dr) + i * g.ld_dr, c, g.cols, g.vec, d[j]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (c + e >= g.cols) { d[j].v[e] = 0.f; continue; }
        d[j].v[e] *= g.alpha;
        sum[0][j].v[e] += d[j].v[e] * u[j].v[e];
        if (gate) d[j].v[e] *= gate[c + e];
        if (g.post != NORM_NONE) {
          sum[1][j].v[e] += d[j].v[e] * f[j].v[e];
          sum[2][j].v[e] += d[j].v[e];
          d[j].v[e] *= g.w_post[c + e];
        }
      }
    }
    if (g.post != NORM_NONE) norm_gradient<NJ>(d, f, inv_f, g.post, g.cols, slot + 40);
#pragma unroll
    for (int j = 0; j < NJ; ++j) store8(static_cast<T *>(g.df) + i * g.ld_df, (at + 256 * j) * 8, g.cols, g.vec, d[j]);
    if (g.dgate && left && --left == 0) {
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int c = (at + 256 * j) * 8 + e;
          if (c < g.cols) g.dgate[group * g.cols + c] = sum[0][j].v[e];
          sum[0][j].v[e] = 0.f;
        }
      left = g.group_rows;
      ++group;
    }
  }
  float *out = g.partial + (int64_t)blockIdx.x * 5 * g.cols;
#pragma unroll
  for (int q = 0; q < 5; ++q) {
    if (q == 0 ? !g.gate || !g.chunks_per_group : q == 1 ? g.post == NORM_NONE : q == 2 ? g.post != NORM_LAYER : q == 3 ? g.pre == NORM_NONE : g.pre != NORM_LAYER) continue;
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int c = (at + 256 * j) * 8 + e;
        if (c < g.cols) out[q * g.cols + c] = sum[q][j].v[e];
      }
  }
}

}  // namespace shampoo
