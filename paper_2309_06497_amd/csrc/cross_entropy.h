// Softmax cross entropy of a linear layer z = x w^T + b over many classes, with its gradients.
//
//   lse_i = log sum_v exp z_iv        loss_i = lse_i - z_{i,t_i}        g_iv = c_i (exp(z_iv - lse_i) - [v = t_i])
//   dx = g w        dw = g^T x        db = column sums of g
//
// c_i = scale weight_i, zero where the target is ignored.  Logits of a piece of the rows at a time lie in scratch.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include "vectors.h"

namespace shampoo {

// lse, loss and c of a row of float32 logits; a workgroup per row.  z += bias on the way.
struct RowLossArgs {
  float *z; int64_t ldz;
  const float *bias; const int64_t *targets; const float *weight;
  float scale;
  float *lse, *coef, *loss;
  int32_t classes;
};
__global__ __launch_bounds__(256) void row_loss_kernel(const RowLossArgs g) {
  __shared__ float red[8];
  const int64_t i = blockIdx.x;
  float *z = g.z + i * g.ldz;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  float m = -INFINITY;
  bool nan = false;
  for (int v = tid; v < g.classes; v += 256) {
    float x = z[v];
    if (g.bias) { x += g.bias[v]; z[v] = x; }
    nan |= x != x;
    m = fmaxf(m, x);
  }
  if (nan) m = NAN;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) { const float y = __shfl_xor(m, o, 64); m = m != m || y != y ? NAN : fmaxf(m, y); }
  if (lane == 0) red[wave] = m;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 4; ++k) { const float y = red[k]; m = m != m || y != y ? NAN : fmaxf(m, y); }
  float s = 0.f;
  const float base = m == -INFINITY ? 0.f : m;
  for (int v = tid; v < g.classes; v += 256) s += expf(z[v] - base);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if (lane == 0) red[4 + wave] = s;
  __syncthreads();
  if (tid != 0) return;
  s = (red[4] + red[5]) + (red[6] + red[7]);
  const float lse = base + logf(s);
  const int64_t t = g.targets[i];
  const bool valid = t >= 0 && t < g.classes;
  g.lse[i] = lse;
  g.coef[i] = valid ? g.scale * (g.weight ? g.weight[i] : 1.f) : 0.f;
  const float zt = valid ? z[t] : 0.f;
  g.loss[i] = !valid ? 0.f : zt == -INFINITY ? INFINITY : lse - zt;
}

// g of a piece of the rows as PLANES bf16 planes [plane][rows][ldg] (ldg: classes rounded up, zeros there), and the column
// sums of every range of rows for the bias.  A thread has eight columns of the rows of its range.
struct SoftmaxGradArgs {
  const float *z; int64_t ldz;
  const float *lse, *coef; const int64_t *targets;
  uint16_t *out; int64_t plane, ldg;
  float *sums;                       // [ranges][classes], or nullptr
  int32_t rows, classes, per_range;
};
template <int PLANES> __global__ __launch_bounds__(256) void softmax_grad_kernel(const SoftmaxGradArgs g) {
  const int c = (blockIdx.x * 256 + threadIdx.x) * 8;
  if (c >= g.ldg) return;
  const int i0 = blockIdx.y * g.per_range, i1 = min(g.rows, i0 + g.per_range);
  f32x8 sum = {{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}};
  for (int i = i0; i < i1; ++i) {
    const float lse = g.lse[i], k = g.coef[i];
    const int64_t t = g.targets[i] - c;
    const f32x8 z = load8(g.z + i * g.ldz, c, g.classes, true);
    uint16_t q[8][PLANES];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float x = 0.f;
      if (k != 0.f && c + e < g.classes && lse != -INFINITY) x = k * (expf(z.v[e] - lse) - (t == e ? 1.f : 0.f));
      sum.v[e] += x;
      bf16_planes_of<PLANES>(x, q[e]);
    }
#pragma unroll
    for (int s = 0; s < PLANES; ++s) {
      uint4 w;
      w.x = q[0][s] | (uint32_t)q[1][s] << 16; w.y = q[2][s] | (uint32_t)q[3][s] << 16;
      w.z = q[4][s] | (uint32_t)q[5][s] << 16; w.w = q[6][s] | (uint32_t)q[7][s] << 16;
      *reinterpret_cast<uint4 *>(g.out + s * g.plane + (int64_t)i * g.ldg + c) = w;
    }
  }
  if (!g.sums) return;
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (c + e < g.classes) g.sums[(int64_t)blockIdx.y * g.classes + c + e] = sum.v[e];
}

}  // namespace shampoo
