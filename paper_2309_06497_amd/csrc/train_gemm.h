// Matrix products of the training operators (cross_entropy.h, checkpoint.h) on the bf16 matrix cores.
//
//   C[m][n] = sum over pairs (s, t) of planes, sum over k: A_s(m, k) B_t(n, k)
//
// Operands are bf16 planes in memory: one for a bf16 matrix, up to three for a float32 one (x = h + l + m, 8 bits each), whose
// products (s, t) are all that float32 accuracy needs, smallest first: one loop over k behind the other.  An operand lies along
// k (ptr[row * ld + k]) or along rows (ptr[k * ld + row]).  Contract, which the host keeps: 16-byte aligned, ld % 8 == 0; along k
// readable up to the next multiple of 64 of K and zero there, along rows readable up to a multiple of 8 of the rows; and where both
// lie along rows, one of them has zeros for k from K to the next multiple of 64 (both: an infinity in the other's last k meets no zero).
//
// Tile of 64 TI x 64 TI per workgroup of four wavefronts, 32 TI x 32 TI each as TI x TI tiles of v_mfma_f32_32x32x16_bf16.  TI = 4:
// 256 accumulator registers, one wavefront per SIMD; 8 KB of operands from LDS per 16 products of 32 cycles, half of what LDS
// delivers (with 128 x 64 per wavefront it would be three quarters, and the loads into LDS take another quarter).  TI = 2 where that gives too
// few workgroups.
//
// Slabs of 64 values of k go straight into LDS (global_load_lds_dwordx4), the next one in flight while one is multiplied.  Such a
// load fills 1 KiB of consecutive LDS, so bank conflicts are kept away by which 16 bytes a lane asks for:
//   along k:    LDS rows of 128 bytes; chunk c of row r at position c ^ (r / 2 % 8).  16 lanes that are served together read one
//               chunk of 16 rows: two rows a 256-byte line, each pair of rows another position.
//   along rows: LDS rows of one k; chunk c (8 rows of the operand) of k at position c ^ 4 (k % 4).  ds_read_b64_tr_b16 hands
//               four values of k of one row to a lane: 16 lanes read 4 k of 16 rows, the four k in four quarters of the banks.
// Past the end of an operand its last row, or last k, is read again: rows for results that nobody keeps, k for products with the
// other operand's zeros.  So every load is one instruction: a scalar base that moves on by a slab, and an offset per lane.
//
// The MFMA operands are handed over swapped, so that a lane has one row of C and runs of four columns: softmax statistics are sums over
// registers, and stores go through LDS in whole rows.
//
// Bound by the matrix cores and the clock that they leave: of 8192 x 2048 x 131072 in bf16, dw runs at 1.17 PFLOP/s (1.24 on a card with a higher clock) with them busy for
// 72 % of the cycles at 1.50 GHz, no bank conflicts, dx at 1.22; the logits at 1.04, since a tile ends with 13 vector
// operations per logit.  8192 x 2048 x 8192 (dw) 1.16.  Small: 256 x 2048 x 1000, six products of planes, 15 ... 19 us a product.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <type_traits>
#include <utility>
#include "lds_dma.h"
#include "vectors.h"

namespace shampoo {

enum { LIE_K = 0, LIE_ROWS = 1 };          // which index of an operand is contiguous
enum { STORE_F32 = 0, STORE_BF16 = 1, STORE_NOTHING = 2 };
// What becomes of a tile: C itself; the logits' statistics and the logits in float32 (or not at all) or in 16 bits; the gradient of the logits
enum { END_PLAIN = 0, END_LOGITS = 1, END_LOGITS_U16 = 2, END_GRAD = 3 };

struct TrainGemmArgs {
  const uint16_t *a, *b;
  int64_t lda, ldb, a_plane, b_plane;      // elements
  int32_t M, N, K;
  int32_t products;                        // pairs of planes
  int32_t padded;                          // both along rows: 1: A has the zeros, 2: B
  uint32_t plane_a, plane_b;               // four bits each: the planes of product i
  int32_t tiles_m, tiles_n, splits, per_split;   // slabs of the whole sequence (products x ceil(K / 64)) per split
  int32_t tile0, tiles;                    // this launch's: tile0 ... tile0 + tiles - 1
  int32_t by_tile;                         // c holds this launch's tiles one behind the other, 64 TI x 64 TI each, per split
  void *c; int64_t ldc, c_split;           // c_split: from the result of a split to the next
  const float *add; int64_t ldadd;         // C += add (float32; may be c itself) or nullptr
  float alpha;                             // C = alpha A B^T + add
  int32_t store;
  // END_LOGITS...: z = C + bias (16 bits: no bias); per row and span (32 TI columns): the largest z and sum of exp(z - largest); the target's z
  const float *bias; const int64_t *targets;
  float2 *stats; int64_t stats_ld;         // [span][row]
  float *target_z;
  // END_GRAD, from the statistics of a first product: share exp(z - top) - coef [target] as bf16 planes
  const float *top, *coef, *share; int64_t c_plane; int32_t c_planes;
};

typedef float train_f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int TG_BK = 64;
// distance of a logit from the largest of its span in 16 bits: steps of 2^-10 in the exponent of 2
constexpr float LOGIT_STEPS = 1024.f, LOG2_E = 1.4426950408889634f;

// two of them, from z - largest
__device__ __forceinline__ uint32_t logit_pair(float d, float e) {
  constexpr float C = -LOG2_E * LOGIT_STEPS / 65535.f;
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pknorm_u16(d * C, e * C));
}

// Where a tile lies: columns of eight tiles, so that neighbours in number share operands.
__device__ __forceinline__ void tile_place(int tile, int tiles_m, int tiles_n, int &tm, int &tn) {
  const int group = tile / (8 * tiles_n), in_group = tile - group * 8 * tiles_n, rows = min(8, tiles_m - 8 * group);
  tm = 8 * group + in_group % rows;
  tn = in_group / rows;
}

// LDS accesses of one wavefront that depend on one another: LDS keeps their order, the compiler must
__device__ __forceinline__ void tg_wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// How a lane fills and reads the slab of one operand of 64 TI rows.
template <int LIE, int TI> struct SlabSide {
  static constexpr int ROWS = 64 * TI, BYTES = ROWS * TG_BK * 2, PIECES = BYTES / 4096;   // 1 KiB pieces per wavefront
  static constexpr int CHUNKS = LIE == LIE_K ? 8 : ROWS / 8;        // 16-byte chunks of an LDS row
  static constexpr int STEP_READS = LIE == LIE_K ? TI : 2 * TI;     // LDS reads for 16 values of k
  uint32_t off[PIECES];        // bytes from the tile's corner
  uint32_t addr[4];            // LDS: along k, one for each 16 values of k; along rows, one for each 32 rows

  // k_left: values of k that are there
  __device__ __forceinline__ void offsets(int64_t ld, int rows_left, int k_left, int wave, int lane) {
#pragma unroll
    for (int q = 0; q < PIECES; ++q) {
      const int p = (wave * PIECES + q) * 64 + lane, r = p / CHUNKS, pos = p % CHUNKS;
      if (LIE == LIE_K) off[q] = (uint32_t)(min(r, rows_left - 1) * ld * 2) + (pos ^ ((r >> 1) & 7)) * 16;
      else off[q] = (uint32_t)(min(r, k_left - 1) * ld * 2) + min(pos ^ (4 * (r & 3)), (rows_left - 1) >> 3) * 16;
    }
  }
  __device__ __forceinline__ void addresses(int side, int lane, uint32_t lds) {
    if (LIE == LIE_K) {
      const int f = lane & 31, q = lane >> 5;
#pragma unroll
      for (int s = 0; s < 4; ++s) addr[s] = lds + (side * 32 * TI + f) * 128 + (((2 * s + q) ^ ((f >> 1) & 7)) * 16);
    } else {
      const int b = lane >> 4, t = lane & 15, k = 8 * (b >> 1) + (t >> 2);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int ch = side * 4 * TI + 4 * (i < TI ? i : 0) + 2 * (b & 1) + ((t & 3) >> 1);
        addr[i] = lds + k * ROWS * 2 + ((ch ^ (4 * (t >> 2))) * 16) + (t & 1) * 8;
      }
    }
  }
};

template <typename F, int... I> __device__ __forceinline__ void tg_each(std::integer_sequence<int, I...>, F &&f) { (f(std::integral_constant<int, I>()), ...); }

#define TG_READ128(dst, addr, imm) asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(dst) : "v"(addr), "n"(imm) : "memory")
#define TG_READ_TR(dst, addr, imm) asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(dst) : "v"(addr), "n"(imm) : "memory")

// One operand of 16 values of k of 32 TI rows: what the matrix cores take.
template <int LIE, int TI> struct SlabRegs {
  u32x4 f[LIE == LIE_K ? TI : 1];
  u32x2 t[LIE == LIE_K ? 1 : TI][2];
  // LDS read number R of step S from the stage at byte `st`
  template <int R, int S> __device__ __forceinline__ void read(const SlabSide<LIE, TI> &side, uint32_t st) {
    if constexpr (LIE == LIE_K) TG_READ128(f[R], side.addr[S] + st, R * 4096);
    else TG_READ_TR(t[R >> 1][R & 1], side.addr[R >> 1] + st, (16 * S + 4 * (R & 1)) * 128 * TI);
  }
  // behind the wait: the compiler may use them from here on
  __device__ __forceinline__ void arrived() {
#pragma unroll
    for (int i = 0; i < TI; ++i) {
      if constexpr (LIE == LIE_K) asm volatile("" : "+v"(f[i])); else asm volatile("" : "+v"(t[i][0]), "+v"(t[i][1]));
    }
  }
  __device__ __forceinline__ bf16x8 operand(int i) const {
    if constexpr (LIE == LIE_K) return __builtin_bit_cast(bf16x8, f[i]);
    else return __builtin_bit_cast(bf16x8, __builtin_shufflevector(t[i][0], t[i][1], 0, 1, 2, 3));
  }
};

// One tile; smem: GEMM_LDS bytes.
template <int TI, int STAGES> constexpr int GEMM_LDS = STAGES * 64 * TI * TG_BK * 2 * 2;
template <int TI, int STAGES, int ALIE, int BLIE, int END>
__device__ __forceinline__ void train_gemm_tile(const TrainGemmArgs &g, int block, unsigned char *smem) {
  typedef SlabSide<ALIE, TI> SideA;
  typedef SlabSide<BLIE, TI> SideB;
  constexpr int TILE = 64 * TI, SPAN = 32 * TI, STAGE = SideA::BYTES + SideB::BYTES, PIECES = SideA::PIECES, NMM = TI * TI;
  const int total = g.tiles * g.splits;
  // an XCD (workgroup index modulo 8) has neighbouring tiles
  const int per = (total + 7) / 8, logical = (block & 7) * per + (block >> 3);
  if (logical >= total || (block >> 3) >= per) return;
  const int split = logical / g.tiles, tile = g.tile0 + logical - split * g.tiles;
  int tm, tn;
  tile_place(tile, g.tiles_m, g.tiles_n, tm, tn);
  const int row0 = tm * TILE, col0 = tn * TILE;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave >> 1, wn = wave & 1;
  const uint32_t lds = (uint32_t)(uintptr_t)(lds_void *)smem;

  SideA sa; SideB sb;
  sa.addresses(wm, lane, lds);
  sb.addresses(wn, lane, lds + SideA::BYTES);
  const uint16_t *corner_a = g.a + (ALIE == LIE_K ? (int64_t)row0 * g.lda : row0), *corner_b = g.b + (BLIE == LIE_K ? (int64_t)col0 * g.ldb : col0);
  const int64_t step_a = ALIE == LIE_K ? TG_BK : TG_BK * g.lda, step_b = BLIE == LIE_K ? TG_BK : TG_BK * g.ldb;
  const int slabs_k = (g.K + TG_BK - 1) / TG_BK, all = slabs_k * g.products;
  const int first = split * g.per_split, count = min(g.per_split, all - first);

  // the slab that is loaded next: where it begins, and how much of k is left there; behind the last one that one again
  int in_q = first / slabs_k, in_s = first - in_q * slabs_k, in_left = count, in_k;
  const char *in_a, *in_b;
  auto locate = [&]() {
    const int pa = (g.plane_a >> (4 * in_q)) & 15, pb = (g.plane_b >> (4 * in_q)) & 15;
    in_a = uniform_ptr(corner_a + pa * g.a_plane + in_s * step_a);
    in_b = uniform_ptr(corner_b + pb * g.b_plane + in_s * step_b);
    in_k = g.K - in_s * TG_BK;
    sa.offsets(g.lda, g.M - row0, g.padded & 1 ? TG_BK : in_k, wave, lane);
    sb.offsets(g.ldb, g.N - col0, g.padded & 2 ? TG_BK : in_k, wave, lane);
  };
  auto next_slab = [&]() {
    if (--in_left > 0) {
      in_a += 2 * step_a; in_b += 2 * step_b;
      in_k -= TG_BK;
      if (in_k < TG_BK) {                          // the end of k, or the next pair of planes
        if (in_k <= 0) { ++in_q; in_s = 0; } else { in_s = slabs_k - 1; }
        locate();
      }
    }
  };
  auto load_a = [&](int q, int stage) {
    __builtin_amdgcn_global_load_lds((glb_void *)(in_a + sa.off[q]), (lds_void *)(smem + stage + (wave * PIECES + q) * 1024), 16, 0, 0);
  };
  auto load_b = [&](int q, int stage) {
    __builtin_amdgcn_global_load_lds((glb_void *)(in_b + sb.off[q]), (lds_void *)(smem + stage + SideA::BYTES + (wave * PIECES + q) * 1024), 16, 0, 0);
  };

  train_f32x16 acc[TI][TI];
#pragma unroll
  for (int i = 0; i < TI; ++i)
#pragma unroll
    for (int j = 0; j < TI; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;

  // two sets that take turns
  SlabRegs<ALIE, TI> ra[2];
  SlabRegs<BLIE, TI> rb[2];
  constexpr int READS = SideA::STEP_READS + SideB::STEP_READS;
  auto read = [&](auto rc, auto sc, uint32_t from) {
    constexpr int R = decltype(rc)::value, S = decltype(sc)::value, B0 = SideA::STEP_READS;
    if constexpr (R < B0) ra[S & 1].template read<R, S>(sa, from);
    else if constexpr (R < READS) rb[S & 1].template read<R - B0, S>(sb, from);
  };

  // One step: the products of 16 values of k, and between them, one at a time, so that the matrix cores do not wait for the wavefront
  // to issue something else, the LDS reads of the next step (in its first half) and loads of slabs to come (in its second).  The loads of
  // slab t + STAGES begin with step 3 of slab t, behind the barrier after which nobody reads its stage any more, and end
  // with step 0 of slab t + 1.  st: the stage of this slab, st_next: of the next one, st_in: of the one that is loaded.
  constexpr int HALF = NMM / 2, PER_SLOT = (READS + HALF - 1) / HALF, LOADS_PER_SLOT = (PIECES + HALF - 1) / HALF;
  auto step = [&](auto sc, uint32_t st, uint32_t st_next, uint32_t st_in) {
    constexpr int S = decltype(sc)::value, X = S & 1, LEAD = S == 3 ? NMM / 8 + (NMM < 8) : 0;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    ra[X].arrived(); rb[X].arrived();
    LDS_SCHED_BARRIER();
    tg_each(std::make_integer_sequence<int, NMM>(), [&](auto mc) {
      constexpr int P = decltype(mc)::value, I = P / TI, J = P % TI;
      acc[I][J] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(rb[X].operand(J), ra[X].operand(I), acc[I][J], 0, 0, 0);
      if constexpr (S == 3 && P == LEAD - 1) {
        LDS_SCHED_BARRIER();
        LDS_DMA_WAIT_VM((STAGES - 2) * 2 * PIECES);       // the next slab is there
        __builtin_amdgcn_s_barrier();
      }
      LDS_SCHED_BARRIER();
      if constexpr (P >= LEAD && P < LEAD + HALF) {
        tg_each(std::make_integer_sequence<int, PER_SLOT>(), [&](auto rc) {
          read(std::integral_constant<int, (P - LEAD) * PER_SLOT + decltype(rc)::value>(), std::integral_constant<int, (S + 1) & 3>(), S == 3 ? st_next : st);
        });
      }
      if constexpr (P >= HALF && (S == 3 || S == 0)) {
#pragma unroll
        for (int q = (P - HALF) * LOADS_PER_SLOT; q < (P - HALF + 1) * LOADS_PER_SLOT && q < PIECES; ++q) {
          if constexpr (S == 3) load_a(q, st_in); else load_b(q, st_in);
        }
      }
      LDS_SCHED_BARRIER();
    });
  };

  locate();
#pragma unroll
  for (int t = 0; t < STAGES; ++t) {
#pragma unroll
    for (int q = 0; q < PIECES; ++q) load_a(q, t * STAGE);
    if (t == STAGES - 1) break;
#pragma unroll
    for (int q = 0; q < PIECES; ++q) load_b(q, t * STAGE);
    next_slab();
  }
  LDS_DMA_WAIT_VM((STAGES - 2) * 2 * PIECES + PIECES);
  __builtin_amdgcn_s_barrier();
  tg_each(std::make_integer_sequence<int, READS>(), [&](auto rc) { read(rc, std::integral_constant<int, 0>(), 0); });
  uint32_t st = 0;
  for (int t = 0; t < count; ++t) {
    const uint32_t next = st + STAGE == STAGES * STAGE ? 0 : st + STAGE, before = st == 0 ? (STAGES - 1) * STAGE : st - STAGE;
    step(std::integral_constant<int, 0>(), st, next, before);
    step(std::integral_constant<int, 1>(), st, next, 0);
    next_slab();
    step(std::integral_constant<int, 2>(), st, next, 0);
    step(std::integral_constant<int, 3>(), st, next, st);
    st = next;
  }
  // the rows' targets in this span (-1: elsewhere), all asked for at once
  [[maybe_unused]] const int colw = col0 + wn * SPAN, roww = row0 + wm * SPAN;
  [[maybe_unused]] int target_at[TI];
  [[maybe_unused]] float row_top[TI], row_coef[TI], row_share[TI];
  if constexpr (END != END_PLAIN) {
#pragma unroll
    for (int i = 0; i < TI; ++i) {
      const int row = min(roww + 32 * i + (lane & 31), g.M - 1);
      const int64_t t = g.targets[row] - colw;
      target_at[i] = t >= 0 && t < SPAN && colw + t < g.N ? (int)t : -1;
      if constexpr (END == END_GRAD) { row_top[i] = g.top[row]; row_coef[i] = g.coef[row]; row_share[i] = g.share[row]; }
    }
  }
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  ra[0].arrived(); rb[0].arrived();
  LDS_DMA_WAIT_VM(0);
  __syncthreads();

  // A lane has row lane % 32 of every tile, columns 8 (v / 4) + 4 (lane / 32) + v % 4.  32 rows at a time go through LDS, which only
  // this wavefront touches.
  constexpr int PITCH = SPAN + 4, PITCH16 = SPAN + 8;      // floats, 16-bit logits: rows are 16-byte aligned and four banks apart
  static_assert(4 * 32 * PITCH * 4 + 4 * SPAN * 4 <= STAGES * STAGE, "LDS");
  float *buf = reinterpret_cast<float *>(smem) + wave * 32 * PITCH;
  const int half = lane >> 5;
  [[maybe_unused]] float *bias = reinterpret_cast<float *>(smem) + 4 * 32 * PITCH + wave * SPAN;
  if constexpr (END == END_LOGITS || END == END_GRAD) {
    for (int j = lane; j < SPAN; j += 64) bias[j] = colw + j >= g.N ? -INFINITY : g.bias ? g.bias[colw + j] : 0.f;   // no class there: probability 0
  }
  constexpr int LANES = SPAN / 8, ROWS_AT_ONCE = 64 / LANES;      // eight columns a lane
  const int c = (lane % LANES) * 8, col = colw + c, limit = END == END_PLAIN ? g.N : (int)g.ldc;
  const int row_limit = END == END_GRAD ? (g.M + TG_BK - 1) / TG_BK * TG_BK : g.M;                  // zeros behind the last row
  // rows r, r + ROWS_AT_ONCE, ... of the 32 that lie in LDS
  auto put = [&](int i, auto &&store) {
    tg_wave_order();
#pragma unroll
    for (int r = lane / LANES; r < 32; r += ROWS_AT_ONCE) {
      const int out = roww + 32 * i + r;
      if (out < row_limit && col < limit) store(r, (int64_t)out);
    }
    tg_wave_order();
  };
  auto stage = [&](int i) {
#pragma unroll
    for (int j = 0; j < TI; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<float4 *>(buf + (lane & 31) * PITCH + 32 * j + 8 * q + 4 * half) =
            make_float4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
  };
  auto staged = [&](int r) { return load8(buf + r * PITCH + c, 0, 8); };

  if constexpr (END == END_PLAIN) {
    const int64_t from = split * g.c_split + (g.by_tile ? (int64_t)(tile - g.tile0) * TILE * TILE - (int64_t)row0 * TILE - col0 : 0);
#pragma unroll
    for (int i = 0; i < TI; ++i) {
      stage(i);
      put(i, [&](int r, int64_t out) {
        f32x8 z = staged(r);
#pragma unroll
        for (int e = 0; e < 8; ++e) z.v[e] *= g.alpha;
        if (g.add) {
          const f32x8 old = load8(g.add + out * g.ldadd, col, g.N);
#pragma unroll
          for (int e = 0; e < 8; ++e) z.v[e] += old.v[e];
        }
        if (g.store == STORE_BF16) store8(static_cast<uint16_t *>(g.c) + out * g.ldc, col, limit, z);
        else store8(static_cast<float *>(g.c) + from + out * g.ldc, col, limit, z);
      });
    }
  } else {
    tg_wave_order();
#pragma unroll
    for (int i = 0; i < TI; ++i) {
      const int row = roww + 32 * i + (lane & 31);
      if constexpr (END == END_LOGITS || END == END_GRAD) {
#pragma unroll
        for (int j = 0; j < TI; ++j)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const float4 b = *reinterpret_cast<const float4 *>(bias + 32 * j + 8 * q + 4 * half);
            acc[i][j][4 * q] += b.x; acc[i][j][4 * q + 1] += b.y; acc[i][j][4 * q + 2] += b.z; acc[i][j][4 * q + 3] += b.w;
          }
      }
      if constexpr (END == END_GRAD) {
        const float top = row_top[i], share = row_share[i], k = row < g.M ? row_coef[i] : 0.f;
        const int at = target_at[i] - 4 * half;
#pragma unroll
        for (int j = 0; j < TI; ++j)
#pragma unroll
          for (int v = 0; v < 16; ++v) {
            const float p = __builtin_amdgcn_exp2f((acc[i][j][v] - top) * LOG2_E);
            acc[i][j][v] = k != 0.f ? fmaf(share, p, at == 32 * j + 8 * (v >> 2) + (v & 3) ? -k : 0.f) : 0.f;
          }
        stage(i);
        put(i, [&](int r, int64_t out) {
          f32x8 z = staged(r);
          uint16_t *to = static_cast<uint16_t *>(g.c) + out * g.ldc + col;
          for (int s = 0; s < g.c_planes; ++s) {          // each plane what the ones before it leave
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              w[e] = bf16_pair(z.v[2 * e], z.v[2 * e + 1]);
              z.v[2 * e] -= __uint_as_float(w[e] << 16); z.v[2 * e + 1] -= __uint_as_float(w[e] & 0xffff0000u);
            }
            *reinterpret_cast<uint4 *>(to + s * g.c_plane) = make_uint4(w[0], w[1], w[2], w[3]);
          }
        });
      } else {
        // ENDS: the span reaches past the last class (float32: the bias has taken care of that)
        auto statistics = [&](auto ends) {
          constexpr bool ENDS = decltype(ends)::value;
          auto z = [&](int j, int v) {
            const float x = acc[i][j][v];
            return ENDS && colw + 32 * j + 8 * (v >> 2) + 4 * half + (v & 3) >= g.N ? -INFINITY : x;
          };
          float largest = -INFINITY;
#pragma unroll
          for (int j = 0; j < TI; ++j)
#pragma unroll
            for (int v = 0; v < 16; v += 2) largest = fmaxf(largest, fmaxf(z(j, v), z(j, v + 1)));
          largest = fmaxf(largest, __shfl_xor(largest, 32, 64));
          const float base = largest == -INFINITY ? 0.f : largest;
          const int target = target_at[i];
          const bool here = target >= 0 && row < g.M;
          if (__any(here)) {
            float zt = 0.f;
#pragma unroll
            for (int j = 0; j < TI; ++j)
#pragma unroll
              for (int v = 0; v < 16; ++v) zt = target == 32 * j + 8 * (v >> 2) + 4 * half + (v & 3) ? acc[i][j][v] : zt;
            if (here && ((target >> 2) & 1) == half) g.target_z[row] = zt;
          }
          // exp of the distance from the largest, and that in 16 bits, one conversion for two
          float sum = 0.f;
#pragma unroll
          for (int j = 0; j < TI; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              float d[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                d[e] = z(j, 4 * q + e) - base;
                sum += __builtin_amdgcn_exp2f(d[e] * LOG2_E);
              }
              if constexpr (END == END_LOGITS_U16) {
                const u32x2 w = {logit_pair(d[0], d[1]), logit_pair(d[2], d[3])};
                *reinterpret_cast<u32x2 *>(reinterpret_cast<uint16_t *>(buf) + (lane & 31) * PITCH16 + 32 * j + 8 * q + 4 * half) = w;
              }
            }
          sum += __shfl_xor(sum, 32, 64);
          if (half == 0 && row < g.M) g.stats[(int64_t)(colw / SPAN) * g.stats_ld + row] = make_float2(largest, sum);
        };
        if constexpr (END == END_LOGITS_U16) {
          if (colw + SPAN > g.N) statistics(std::true_type()); else statistics(std::false_type());
          put(i, [&](int r, int64_t out) {
            *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(g.c) + out * g.ldc + col) =
                *reinterpret_cast<const uint4 *>(reinterpret_cast<const uint16_t *>(buf) + r * PITCH16 + c);
          });
        } else {
          statistics(std::false_type());
          if (g.store != STORE_NOTHING) {
            stage(i);
            put(i, [&](int r, int64_t out) { store8(static_cast<float *>(g.c) + out * g.ldc, col, limit, staged(r)); });
          }
        }
      }
    }
  }
}

template <int TI, int STAGES, int ALIE, int BLIE, int END>
__global__ __launch_bounds__(256, TI == 2 && STAGES == 2 ? 2 : 1) void train_gemm_kernel(const TrainGemmArgs g) {
  __shared__ __align__(256) unsigned char smem[GEMM_LDS<TI, STAGES>];
  train_gemm_tile<TI, STAGES, ALIE, BLIE, END>(g, (int)blockIdx.x, smem);
}

// Two small products that do not depend on one another, in one launch: the first `blocks` workgroups (a multiple of 8) have g, whose A
// lies along k, the others h, whose operands both lie along rows.
template <int STAGES, int BLIE> __global__ __launch_bounds__(256, STAGES == 2 ? 2 : 1) void train_gemm_pair_kernel(const TrainGemmArgs g, const TrainGemmArgs h, int blocks) {
  __shared__ __align__(256) unsigned char smem[GEMM_LDS<2, STAGES>];
  const int block = (int)blockIdx.x;
  if (block < blocks) train_gemm_tile<2, STAGES, LIE_K, BLIE, END_PLAIN>(g, block, smem);
  else train_gemm_tile<2, STAGES, LIE_ROWS, LIE_ROWS, END_PLAIN>(h, block - blocks, smem);
}

// The results of several splits, float32 [split][rows][cols], added up in an order that does not depend on the launch.  LANES
// threads share a piece of eight columns where there are many splits, so that their loads are on their way together.
// Workgroups from `blocks` on add up the rows of `sums` (16 columns each, 16 threads a column), which saves a launch of their own.
struct RowSums { const float *in; float *out; int32_t parts, cols, add; };      // [parts][cols]; add: to what is there
struct JoinArgs {
  const float *part; int64_t stride; int32_t splits;
  void *c; int64_t ldc; const float *add; int64_t ldadd;
  int64_t row0; uint32_t pieces, per_row;
  int32_t cols, pitch, store;
  float alpha;
  uint32_t blocks; RowSums sums;
};
__device__ __forceinline__ void row_sums(const RowSums &g, int block) {
  __shared__ float part[16][16];
  const int c = threadIdx.x & 15, k = threadIdx.x >> 4, j = block * 16 + c;
  float s[4] = {0.f, 0.f, 0.f, 0.f};
  if (j < g.cols) {
    const float *p = g.in + j;
    int i = k;
    for (; i + 48 < g.parts; i += 64) {
#pragma unroll
      for (int q = 0; q < 4; ++q) s[q] += p[(int64_t)(i + 16 * q) * g.cols];
    }
    for (; i < g.parts; i += 16) s[0] += p[(int64_t)i * g.cols];
  }
  part[k][c] = (s[0] + s[1]) + (s[2] + s[3]);
  __syncthreads();
  if (k != 0 || j >= g.cols) return;
  float t = 0.f;
#pragma unroll
  for (int q = 0; q < 16; ++q) t += part[q][c];
  g.out[j] = g.add ? g.out[j] + t : t;
}
template <int LANES> __global__ __launch_bounds__(256) void train_join_kernel(const JoinArgs g) {
  if (blockIdx.x >= g.blocks) { row_sums(g.sums, blockIdx.x - g.blocks); return; }
  const uint32_t at = blockIdx.x * (256u / LANES) + threadIdx.x / LANES, i = min(at, g.pieces - 1);
  const int lane = threadIdx.x % LANES;
  const uint32_t r = i / g.per_row;
  const int c = (int)(i - r * g.per_row) * 8;
  const int64_t row = g.row0 + r;
  f32x8 s = {{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}};
#pragma unroll 4
  for (int k = lane; k < g.splits; k += LANES) {
    const f32x8 x = load8(g.part + k * g.stride + row * g.pitch, c, g.pitch);
#pragma unroll
    for (int e = 0; e < 8; ++e) s.v[e] += x.v[e];
  }
#pragma unroll
  for (int o = 1; o < LANES; o <<= 1)
#pragma unroll
    for (int e = 0; e < 8; ++e) s.v[e] += __shfl_xor(s.v[e], o, 64);
  if (at >= g.pieces || lane != 0) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) s.v[e] *= g.alpha;
  if (g.add) {
    const f32x8 x = load8(g.add + row * g.ldadd, c, g.cols);
#pragma unroll
    for (int e = 0; e < 8; ++e) s.v[e] += x.v[e];
  }
  if (g.store == STORE_BF16) store8(static_cast<uint16_t *>(g.c) + row * g.ldc, c, g.cols, s);
  else store8(static_cast<float *>(g.c) + row * g.ldc, c, g.cols, s);
}

// The tiles of a product's last round, which its splits left one behind the other (by_tile), added up in order.
struct JoinTilesArgs {
  const float *part; int64_t stride; int32_t splits;
  void *c; int64_t ldc; const float *add; int64_t ldadd;
  int32_t M, N, tiles_m, tiles_n, tile0, tile, store;       // tile: rows of one
  float alpha;
};
__global__ __launch_bounds__(256) void train_join_tiles_kernel(const JoinTilesArgs g) {
  const int pieces = g.tile * g.tile / 8, per = pieces / 256;           // workgroups of a tile
  const int t = blockIdx.x / per, i = (blockIdx.x - t * per) * 256 + threadIdx.x, r = i / (g.tile / 8), c = (i - r * (g.tile / 8)) * 8;
  int tm, tn;
  tile_place(g.tile0 + t, g.tiles_m, g.tiles_n, tm, tn);
  const int64_t row = (int64_t)tm * g.tile + r;
  const int col = tn * g.tile + c;
  if (row >= g.M || col >= g.N) return;
  const float *p = g.part + (int64_t)t * g.tile * g.tile + (int64_t)i * 8;
  f32x8 s = load8(p, 0, 8);
#pragma unroll 4
  for (int k = 1; k < g.splits; ++k) {
    const f32x8 x = load8(p + k * g.stride, 0, 8);
#pragma unroll
    for (int e = 0; e < 8; ++e) s.v[e] += x.v[e];
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) s.v[e] *= g.alpha;
  if (g.add) {
    const f32x8 x = load8(g.add + row * g.ldadd, col, g.N);
#pragma unroll
    for (int e = 0; e < 8; ++e) s.v[e] += x.v[e];
  }
  if (g.store == STORE_BF16) store8(static_cast<uint16_t *>(g.c) + row * g.ldc, col, g.N, s);
  else store8(static_cast<float *>(g.c) + row * g.ldc, col, g.N, s);
}

}  // namespace shampoo
