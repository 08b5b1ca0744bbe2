// Matrix products of the training operators (cross_entropy.h, checkpoint.h) on the bf16 matrix cores.
//
//   C[m][n] = sum over pairs (s, t) of planes, sum over k: A_s(m, k) B_t(n, k)
//
// Operands are bf16 planes in memory: one for a bf16 matrix, up to three for a float32 one (x = h + l + m, 8 bits each), whose
// products (s, t) are all that float32 accuracy needs, smallest first.  An operand lies along k (ptr[row * ld + k]) or along
// rows (ptr[k * ld + row]).  Contract, which the host keeps: 16-byte aligned, ld % 8 == 0, the contiguous extent readable up to a
// multiple of 8, and zero there where that extent is k.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include "lds_dma.h"

namespace shampoo {

enum { LIE_K = 0, LIE_ROWS = 1 };          // which index of an operand is contiguous
enum { STORE_F32 = 0, STORE_BF16 = 1 };

struct TrainGemmArgs {
  const uint16_t *a, *b;
  int64_t lda, ldb, a_plane, b_plane;      // elements
  int32_t M, N, K;
  int32_t products;                        // pairs of planes
  uint32_t plane_a, plane_b;               // four bits each: the planes of product i
  void *c; int64_t ldc;
  const float *add; int64_t ldadd;         // C += add (float32; may be c itself) or nullptr
  int32_t store;                           // STORE_F32 / STORE_BF16
};

typedef float train_f16 __attribute__((ext_vector_type(16)));

// One 64 x 64 tile per workgroup of four wavefronts (32 x 32 each), 32 values of k at a time through LDS.
template <int ALIE, int BLIE>
__global__ __launch_bounds__(256) void train_gemm_kernel(const TrainGemmArgs g) {
  __shared__ __align__(16) uint16_t as[64][40], bs[64][40];
  const int tiles_n = (g.N + 63) / 64, tm = blockIdx.x / tiles_n, tn = blockIdx.x - tm * tiles_n;
  const int row0 = tm * 64, col0 = tn * 64, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wm = wave >> 1, wn = wave & 1;
  train_f16 acc;
#pragma unroll
  for (int v = 0; v < 16; ++v) acc[v] = 0.f;
  for (int q = 0; q < g.products; ++q) {
    const uint16_t *pa = g.a + (int64_t)((g.plane_a >> (4 * q)) & 15) * g.a_plane, *pb = g.b + (int64_t)((g.plane_b >> (4 * q)) & 15) * g.b_plane;
    for (int k0 = 0; k0 < g.K; k0 += 32) {
      __syncthreads();
      for (int e = tid; e < 64 * 32; e += 256) {
        const int i = ALIE == LIE_K ? e >> 5 : e & 63, k = ALIE == LIE_K ? e & 31 : e >> 6;
        uint16_t v = 0;
        if (row0 + i < g.M && k0 + k < g.K) v = ALIE == LIE_K ? pa[(int64_t)(row0 + i) * g.lda + k0 + k] : pa[(int64_t)(k0 + k) * g.lda + row0 + i];
        as[i][k] = v;
      }
      for (int e = tid; e < 64 * 32; e += 256) {
        const int i = BLIE == LIE_K ? e >> 5 : e & 63, k = BLIE == LIE_K ? e & 31 : e >> 6;
        uint16_t v = 0;
        if (col0 + i < g.N && k0 + k < g.K) v = BLIE == LIE_K ? pb[(int64_t)(col0 + i) * g.ldb + k0 + k] : pb[(int64_t)(k0 + k) * g.ldb + col0 + i];
        bs[i][k] = v;
      }
      __syncthreads();
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const bf16x8 x = *reinterpret_cast<const bf16x8 *>(&as[wm * 32 + (lane & 31)][16 * s + 8 * (lane >> 5)]);
        const bf16x8 y = *reinterpret_cast<const bf16x8 *>(&bs[wn * 32 + (lane & 31)][16 * s + 8 * (lane >> 5)]);
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, y, acc, 0, 0, 0);
      }
    }
  }
  // accumulator element v: row 8 (v / 4) + 4 (lane / 32) + v % 4, column lane % 32
#pragma unroll
  for (int v = 0; v < 16; ++v) {
    const int i = row0 + wm * 32 + 8 * (v >> 2) + 4 * (lane >> 5) + (v & 3), j = col0 + wn * 32 + (lane & 31);
    if (i >= g.M || j >= g.N) continue;
    float x = acc[v];
    if (g.add) x += g.add[(int64_t)i * g.ldadd + j];
    if (g.store == STORE_F32) static_cast<float *>(g.c)[(int64_t)i * g.ldc + j] = x;
    else static_cast<__bf16 *>(g.c)[(int64_t)i * g.ldc + j] = (__bf16)x;
  }
}

}  // namespace shampoo
