// Softmax cross entropy of a linear layer z = x w^T + b over many classes, with its gradients.
//
//   m_i = max_v z_iv        s_i = sum_v exp(z_iv - m_i)        loss_i = (m_i - z_{i,t_i}) + log s_i        g_iv = c_i (exp(z_iv - m_i) / s_i - [v = t_i])
//   dx = g w        dw = g^T x        db = column sums of g
//
// m and log s are never added: beside an m of 1e4 a float32 keeps log s to 5e-4, and that would be the relative error of every p of the row (300 equal
// logits of 1e6: the sum of p 1.016).  z - m is exact where p matters.  A row is kept as m_i, c_i and c_i / s_i, so that g is one fused multiply-add.
//
// c_i = scale weight_i, zero where the target is ignored.  g is kept with the power of two of `scale` alone, and the products' results are
// multiplied by the rest in float32: g of the target is about -c_i in every row, and its rounding to bf16 would be the same error of up
// to 3.9e-3 in all rows, while 1 - p rounds exactly or nearly so (255 x 256 x 20000 at a scale of 1/255: gradients 4.2e-3 off the definition's
// with the scale in g, 1.7 ... 2.0e-3 so, of which 1.7e-3 is the rounding of the result).
// The product that makes z (train_gemm.h) leaves, for every row
// and span of 64 or 128 classes, the largest z and the sum of exp(z - largest), and of a piece of the rows
//   bf16 x, bf16 dw, no bias: the distance of z from the largest of its span in 16 bits, steps of 2^-10 in the exponent of 2
//     (2 bytes per logit; exp(z) is off by 3.4e-4 of itself at most where the rounding of g to bf16 is 3.9e-3; what is further than 64
//     steps of 1 away, 5e-20 of the largest, counts as zero).  g takes its place.
//   float32 x or dw, or a bias: z in float32, beside it g as the bf16 planes that float32 results need.
// Few features (and no sums for a bias): neither; the product runs a second time, once the rows' sums are known, and leaves g itself.
// The three products are 6 rows features classes operations; what lies between them is bound by memory.  8192 x 2048 x 131072 in bf16:
// products 4.24, 3.62 (dx) and 3.75 ms (dw), 16-bit logits to g 0.87 (4.3 GB, 4.9 TB/s), the rows' sums 0.03.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include "train_gemm.h"
#include "vectors.h"

namespace shampoo {

// Logits from the float32 results of several splits of their product, where that has too few tiles to fill the GPU otherwise: what
// the logits' product leaves (train_gemm.h), in spans of 64 classes.  A thread has eight classes of a row and
// every fourth split.
struct LogitsJoinArgs {
  const float *part; int64_t stride, pitch; int32_t splits;
  void *z; int64_t ldz; int32_t end, store;
  const float *bias; const int64_t *targets;
  float2 *stats; int64_t stats_ld; float *target_z;
  int32_t rows, classes;
  uint32_t pieces, per_row;          // ldz / 8, a multiple of 8
};
__global__ __launch_bounds__(256) void logits_join_kernel(const LogitsJoinArgs g) {
  // lanes 8 l ... 8 l + 7 of a span's 32: splits l, l + 4, ...
  const uint32_t piece = (blockIdx.x * 256u + threadIdx.x) / 32 * 8 + (threadIdx.x & 7), at = min(piece, g.pieces - 1);   // the last one again: whole wavefronts
  const int i = at / g.per_row, c = (at - i * g.per_row) * 8, lane = (threadIdx.x >> 3) & 3;
  f32x8 z = {{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}};
#pragma unroll 4
  for (int k = lane; k < g.splits; k += 4) {
    const f32x8 x = load8(g.part + k * g.stride + (int64_t)i * g.pitch, c, (int)g.pitch);
#pragma unroll
    for (int e = 0; e < 8; ++e) z.v[e] += x.v[e];
  }
#pragma unroll
  for (int o = 8; o < 32; o <<= 1)
#pragma unroll
    for (int e = 0; e < 8; ++e) z.v[e] += __shfl_xor(z.v[e], o, 64);
  if (g.bias) {
    const f32x8 b = load8(g.bias, c, g.classes);
#pragma unroll
    for (int e = 0; e < 8; ++e) z.v[e] += b.v[e];
  }
  float largest = -INFINITY;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if (c + e >= g.classes) z.v[e] = -INFINITY;
    largest = fmaxf(largest, z.v[e]);
  }
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) largest = fmaxf(largest, __shfl_xor(largest, o, 64));
  const float base = largest == -INFINITY ? 0.f : largest;
  const int64_t t = g.targets[i] - c;
  float sum = 0.f;
  uint32_t w[4];
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    const float d = z.v[e] - base, d1 = z.v[e + 1] - base;
    sum += __builtin_amdgcn_exp2f(d * LOG2_E) + __builtin_amdgcn_exp2f(d1 * LOG2_E);
    w[e >> 1] = logit_pair(d, d1);
  }
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) sum += __shfl_xor(sum, o, 64);
  if (piece >= g.pieces || lane != 0) return;
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (t == e && c + e < g.classes) g.target_z[i] = z.v[e];
  if ((c & 63) == 0) g.stats[(int64_t)(c >> 6) * g.stats_ld + i] = make_float2(largest, sum);
  if (g.end == END_LOGITS_U16) *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(g.z) + (int64_t)i * g.ldz + c) = make_uint4(w[0], w[1], w[2], w[3]);
  else if (g.store != STORE_NOTHING) store8(static_cast<float *>(g.z) + (int64_t)i * g.ldz, c, (int)g.ldz, z);
}

// m, c, c / s and the loss of every row from the largest logits and sums of its spans: 16 rows per workgroup, 64 threads a row.
struct RowLossArgs {
  const float2 *stats; int64_t stats_ld;
  const float *target_z; const int64_t *targets; const float *weight;
  float scale;
  float *top, *coef, *share, *loss;  // m, c, c / s
  int32_t rows, classes, spans;
};
// exp sums (m, s) and (n, t) together; s is 0 or NaN where m is -infinity
__device__ __forceinline__ void join_exp(float &m, float &s, float n, float t) {
  const float top = fmaxf(m, n);
  const float a = m == -INFINITY ? s : s * __builtin_amdgcn_exp2f((m - top) * LOG2_E), b = n == -INFINITY ? t : t * __builtin_amdgcn_exp2f((n - top) * LOG2_E);
  m = top; s = a + b;
}
// No class left (s = 0): c = 0.
__device__ __forceinline__ void row_end(const RowLossArgs &g, int i, float m, float s, float &top, float &coef, float &share) {
  const int64_t t = g.targets[i];
  const bool valid = t >= 0 && t < g.classes;
  top = m == -INFINITY ? 0.f : m;
  coef = valid && s != 0.f ? g.scale * (g.weight ? g.weight[i] : 1.f) : 0.f;
  share = coef / s;
  const float zt = valid ? g.target_z[i] : 0.f;
  g.loss[i] = !valid ? 0.f : zt == -INFINITY ? INFINITY : (m - zt) + logf(s);
}
__global__ __launch_bounds__(1024) void row_loss_kernel(const RowLossArgs g) {
  __shared__ float2 part[16][16];
  const int r = threadIdx.x & 15, k = threadIdx.x >> 4, i = blockIdx.x * 16 + r;
  float m = -INFINITY, s = 0.f;
  if (i < g.rows) {
#pragma unroll 4
    for (int p = k; p < g.spans; p += 64) {
      const float2 x = g.stats[p * g.stats_ld + i];
      join_exp(m, s, x.x, x.y);
    }
  }
#pragma unroll
  for (int o = 16; o < 64; o <<= 1) {            // the four of a wavefront, then the wavefronts in order
    const float n = __shfl_xor(m, o, 64), t = __shfl_xor(s, o, 64);
    join_exp(m, s, n, t);
  }
  if ((k & 3) == 0) part[k >> 2][r] = make_float2(m, s);
  __syncthreads();
  if (k != 0 || i >= g.rows) return;
  for (int p = 1; p < 16; ++p) join_exp(m, s, part[p][r].x, part[p][r].y);
  row_end(g, i, m, s, g.top[i], g.coef[i], g.share[i]);
}

// g of a piece of the rows, zeros from classes to ldg and in the rows from `rows` to the next multiple of 64.  A thread has eight columns of the rows of its range.
struct SoftmaxGradArgs {
  RowLossArgs row;
  const float *z; int64_t ldg;       // float32 logits
  int32_t span;
  uint16_t *out; int64_t plane;      // [plane][rows][ldg]; 16-bit logits are read here
  float *sums;                       // [ranges][classes] column sums of g, or nullptr; times `alpha`
  int32_t per_range;                 // at most 64
  float alpha;
};
// PLANES = 0: one plane, in the place of 16-bit logits.  Four rows are on their way together.  Where a workgroup has the rows' whole
// width (up to 2048 classes) it ends the rows' sums too: one launch instead of two.
template <int PLANES> __global__ __launch_bounds__(256) void softmax_grad_kernel(const SoftmaxGradArgs g) {
  constexpr int OUT = PLANES ? PLANES : 1, AHEAD = 4;
  __shared__ float row_top[64], row_coef[64], row_share[64];
  const int c = (blockIdx.x * 256 + threadIdx.x) * 8, rows = g.row.rows, classes = g.row.classes;
  const int end = (rows + 63) & ~63, i0 = blockIdx.y * g.per_range, i1 = min(end, i0 + g.per_range);
  {
    const int r = threadIdx.x >> 2, i = i0 + r;                 // four threads a row
    float top = 0.f, coef = 0.f, share = 0.f;                   // nothing behind the last row
    if (gridDim.x == 1) {
      float m = -INFINITY, s = 0.f;
      if (i < min(i1, rows))
        for (int p = threadIdx.x & 3; p < g.row.spans; p += 4) {
          const float2 x = g.row.stats[p * g.row.stats_ld + i];
          join_exp(m, s, x.x, x.y);
        }
#pragma unroll
      for (int o = 1; o < 4; o <<= 1) {
        const float n = __shfl_xor(m, o, 64), t = __shfl_xor(s, o, 64);
        join_exp(m, s, n, t);
      }
      if ((threadIdx.x & 3) == 0 && i < min(i1, rows)) row_end(g.row, i, m, s, top, coef, share);
    } else if (i < min(i1, rows)) { top = g.row.top[i]; coef = g.row.coef[i]; share = g.row.share[i]; }
    if ((threadIdx.x & 3) == 0) { row_top[r] = top; row_coef[r] = coef; row_share[r] = share; }
  }
  __syncthreads();
  if (c >= g.ldg) return;
  const int64_t span = (int64_t)(c / g.span) * g.row.stats_ld;
  f32x8 sum = {{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}};
  for (int first = i0; first < i1; first += AHEAD) {
    Raw8<float> z[PLANES ? AHEAD : 1];
    Raw8<uint16_t> q16[PLANES ? 1 : AHEAD];
    float m[AHEAD], k[AHEAD], share[AHEAD], top[AHEAD];      // top: of the span
    int64_t t[AHEAD];
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
      const int i = min(first + a, i1 - 1);
      const int64_t at = (int64_t)i * g.ldg + c;
      const bool there = i < rows;
      m[a] = row_top[i - i0]; k[a] = row_coef[i - i0]; share[a] = row_share[i - i0]; t[a] = (there ? g.row.targets[i] : 0) - c;
      if constexpr (PLANES == 0) { q16[a] = raw_load8(g.out + at, 0, 8); top[a] = there ? g.row.stats[span + i].x : 0.f; }
      else z[a] = raw_load8(g.z + at, 0, 8);
    }
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
      if (first + a >= i1) break;
      f32x8 p;
      if constexpr (PLANES == 0) {
        const float from = (top[a] - m[a]) * LOG2_E;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t q = (q16[a].u[0][e >> 1] >> (16 * (e & 1))) & 0xffffu;
          p.v[e] = q == 65535u ? 0.f : __builtin_amdgcn_exp2f(from - (float)q * (1.f / LOGIT_STEPS));
        }
      } else {
        p = expand8(z[a]);
#pragma unroll
        for (int e = 0; e < 8; ++e) p.v[e] = expf(p.v[e] - m[a]);
      }
      uint16_t q[8][OUT];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float x = 0.f;
        if (k[a] != 0.f && c + e < classes) x = fmaf(share[a], p.v[e], t[a] == e ? -k[a] : 0.f);
        sum.v[e] += x;
        bf16_planes_of<OUT>(x, q[e]);
      }
#pragma unroll
      for (int s = 0; s < OUT; ++s) {
        uint4 w;
        w.x = q[0][s] | (uint32_t)q[1][s] << 16; w.y = q[2][s] | (uint32_t)q[3][s] << 16;
        w.z = q[4][s] | (uint32_t)q[5][s] << 16; w.w = q[6][s] | (uint32_t)q[7][s] << 16;
        *reinterpret_cast<uint4 *>(g.out + s * g.plane + (int64_t)(first + a) * g.ldg + c) = w;
      }
    }
  }
  if (!g.sums) return;
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (c + e < classes) g.sums[(int64_t)blockIdx.y * classes + c + e] = g.alpha * sum.v[e];
}

}  // namespace shampoo
