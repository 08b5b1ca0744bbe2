// libshampoo, the operators of a training pass: argument checks, workspace layout, kernel launches and the extern "C"
// boundary of their part of shampoo.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "../../include/shampoo.h"
#include "checkpoint.h"
#include "cross_entropy.h"
#include "residual_norm.h"
#include "train_gemm.h"
#include "vectors.h"

using namespace shampoo;

namespace {

constexpr size_t ALIGN = 256;
constexpr int64_t MAX_ROWS = 0x7fffffff;
constexpr int32_t MAX_FEATURES = 65536, MAX_OUT = 1 << 22, MAX_PACKED_COLS = 1 << 20, MAX_NORM_COLS = 16384;
constexpr int64_t MAX_LD = 1 << 22;                        // of an operand as it lies: offsets inside a tile have 32 bits
constexpr size_t LOGIT_BYTES = (size_t)4 << 30;            // scratch of a piece of the rows
constexpr size_t PLANE_BYTES = (size_t)1 << 30;
constexpr int LOGIT_SPLITS = 64;
constexpr int64_t PIECE_ROWS = 256, MAX_PIECE_ROWS = 1 << 21;   // rows of a piece are a multiple of the first (grids: at most 65535 ranges of 64)
constexpr int64_t MAX_TILES = 1 << 23;                     // of a product: threads of a launch have 32 bits
constexpr int64_t MAX_SUM_BLOCKS = 1 << 22;                // workgroups of column sums, beside as many for planes

inline size_t align_up(size_t x) { return (x + ALIGN - 1) / ALIGN * ALIGN; }
inline int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }
inline bool aligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
inline bool dtype_ok(int32_t d) { return d == SHAMPOO_GRAD_F32 || d == SHAMPOO_GRAD_BF16; }
inline int64_t size_of(int32_t d) { return d == SHAMPOO_GRAD_F32 ? 4 : 2; }

#define HIP_TRY(expr)                          \
  do {                                         \
    hipError_t e_ = (expr);                    \
    if (e_ != hipSuccess) return SHAMPOO_ERR_HIP; \
  } while (0)
#define TRY(...)                               \
  do {                                         \
    const int rc_ = (__VA_ARGS__);             \
    if (rc_ != SHAMPOO_OK) return rc_;         \
  } while (0)

// ---------------------------------------------------------------------------
// Workspaces: arrays one behind the other
// ---------------------------------------------------------------------------
struct Arena {
  unsigned char *base; size_t used = 0;
  explicit Arena(void *p) : base(static_cast<unsigned char *>(p)) {}
  template <typename T> T *take(size_t count) {
    T *p = reinterpret_cast<T *>(base + used);
    used += align_up(count * sizeof(T));
    return p;
  }
};
inline int workspace_ok(const void *p, size_t have, size_t want) {
  return want > 0 && (!p || !aligned(p, ALIGN) || have < want) ? SHAMPOO_ERR_WORKSPACE : SHAMPOO_OK;
}

// ---------------------------------------------------------------------------
// Elementwise launches
// ---------------------------------------------------------------------------
// Rows of `per_row` pieces each, at most 2^30 pieces in a launch.
template <typename Launch> int by_rows(int64_t rows, uint32_t per_row, Launch &&launch) {
  const int64_t at_once = std::max<int64_t>(1, ((int64_t)1 << 30) / per_row);
  for (int64_t r = 0; r < rows; r += at_once) {
    const uint32_t pieces = (uint32_t)(std::min(at_once, rows - r) * per_row);
    launch(r, pieces, dim3((pieces + 255) / 256));
    HIP_TRY(hipGetLastError());
  }
  return SHAMPOO_OK;
}

Packed packed_view(const void *p, int64_t rows, int32_t cols) {
  Packed v;
  v.rows = rows; v.cols = cols; v.pitch = (int32_t)round_up(cols, 32);
  v.codes = static_cast<int8_t *>(const_cast<void *>(p));
  v.exps = p ? reinterpret_cast<uint8_t *>(v.codes) + align_up((size_t)rows * v.pitch) : nullptr;
  return v;
}

// bf16 planes of a matrix or of a(checkpoint): what planes_kernel has to do for it
struct PlanesTask { PlanesArgs g; int from, planes; int64_t rows; };
template <typename F> void planes_variant(const PlanesTask &t, F &&f) {
  if (t.from == FROM_F32) f(std::integral_constant<int, FROM_F32>(), std::integral_constant<int, 3>());
  else if (t.from == FROM_BF16) f(std::integral_constant<int, FROM_BF16>(), std::integral_constant<int, 1>());
  else if (t.planes == 1) f(std::integral_constant<int, FROM_PACKED>(), std::integral_constant<int, 1>());
  else f(std::integral_constant<int, FROM_PACKED>(), std::integral_constant<int, 3>());
}
struct ColumnSums {                    // none: parts = 0
  ColumnSumsArgs g; int64_t parts;
  uint32_t blocks() const { return (uint32_t)(parts * ((g.cols + 63) / 64)); }
};
// sums: go along with the first launch
int launch_planes(PlanesTask t, hipStream_t s, ColumnSums sums = {}) {
  t.g.per_row = (uint32_t)(t.g.ld / 8);
  return by_rows(t.rows, t.g.per_row, [&](int64_t r, uint32_t pieces, dim3 grid) {
    t.g.row0 = r; t.g.pieces = pieces;
    const uint32_t more = sums.blocks();
    sums.parts = 0;
    planes_variant(t, [&](auto from, auto planes) {
      constexpr int FROM = decltype(from)::value, PLANES = decltype(planes)::value;
      if constexpr (FROM == FROM_PACKED) {
        if (more) { planes_kernel<FROM, PLANES, true><<<dim3(grid.x + more), 256, 0, s>>>(t.g, grid.x, sums.g); return; }
      }
      planes_kernel<FROM, PLANES, false><<<grid, 256, 0, s>>>(t.g, grid.x, {});
    });
  });
}
// Two of them, in one launch where both are small: up to 2^22 pieces of eight together a launch's latency counts.  g of FROM_F32 with h of the same,
// FROM_BF16 likewise, or g of FROM_PACKED with either.
int launch_planes(PlanesTask g, PlanesTask h, hipStream_t s, const ColumnSums &sums = {}) {
  g.g.per_row = (uint32_t)(g.g.ld / 8); h.g.per_row = (uint32_t)(h.g.ld / 8);
  const int64_t pg = g.rows * g.g.per_row, ph = h.rows * h.g.per_row;
  if (pg + ph > (1 << 22)) { TRY(launch_planes(h, s)); return launch_planes(g, s, sums); }
  g.g.pieces = (uint32_t)pg; h.g.pieces = (uint32_t)ph;
  const uint32_t blocks = (uint32_t)((pg + 255) / 256), from_here = blocks + (uint32_t)((ph + 255) / 256);
  const dim3 all(from_here + sums.blocks());
  planes_variant(h, [&](auto from, auto planes) {
    constexpr int FROM = decltype(from)::value, PLANES = decltype(planes)::value;
    if constexpr (FROM != FROM_PACKED) {
      if (g.from != FROM_PACKED) planes_pair_kernel<FROM, PLANES, FROM, PLANES><<<all, 256, 0, s>>>(g.g, h.g, blocks, from_here, sums.g);
      else if (g.planes == 1) planes_pair_kernel<FROM_PACKED, 1, FROM, PLANES><<<all, 256, 0, s>>>(g.g, h.g, blocks, from_here, sums.g);
      else planes_pair_kernel<FROM_PACKED, 3, FROM, PLANES><<<all, 256, 0, s>>>(g.g, h.g, blocks, from_here, sums.g);
    }
  });
  HIP_TRY(hipGetLastError());
  return SHAMPOO_OK;
}

// outputs[o][j] = sum of the parts of each of `count` entries of g
int launch_join_sums(JoinSumsArgs g, int count, int64_t outputs, hipStream_t s) {
  for (int64_t o = 0; count > 0 && o < outputs; o += 65535) {
    join_sums_kernel<<<dim3((g.cols + 63) / 64, (unsigned)std::min<int64_t>(outputs - o, 65535), count), 1024, 0, s>>>(g);
    HIP_TRY(hipGetLastError());
    for (int k = 0; k < count; ++k) { g.in[k] += 65535 * g.output_stride; g.out[k] += 65535 * g.out_stride; }
  }
  return SHAMPOO_OK;
}
// nothing where `out` is null: a join before it has done it
int launch_row_sums(const RowSums &r, hipStream_t s) {
  JoinSumsArgs g = {};
  g.in[0] = r.in; g.out[0] = r.out; g.parts[0] = r.parts; g.part_stride = r.cols; g.cols = r.cols; g.add = r.add;
  return launch_join_sums(g, r.out ? 1 : 0, 1, s);
}

__global__ __launch_bounds__(256) void zero_rows_kernel(unsigned char *p, int64_t row_bytes, int64_t ld_bytes) {
  for (int64_t j = blockIdx.x * 256 + threadIdx.x; j < row_bytes; j += (int64_t)gridDim.x * 256) p[(int64_t)blockIdx.y * ld_bytes + j] = 0;
}
// gradients of no rows at all
int launch_zero(void *p, int64_t rows, int64_t cols, int64_t ld, int64_t elem, hipStream_t s) {
  for (int64_t r = 0; r < rows; r += 65535) {
    zero_rows_kernel<<<dim3((unsigned)std::min<int64_t>(1024, (cols * elem + 255) / 256), (unsigned)std::min<int64_t>(65535, rows - r)), 256, 0, s>>>(
        static_cast<unsigned char *>(p) + r * ld * elem, cols * elem, ld * elem);
    HIP_TRY(hipGetLastError());
  }
  return SHAMPOO_OK;
}

// ---------------------------------------------------------------------------
// Matrix products
// ---------------------------------------------------------------------------
struct Operand {
  const uint16_t *p; int64_t ld, plane; int planes, lie;
  bool padded = false;       // along rows: zeros behind the last k
};
struct Result {
  void *c; int64_t ldc; int store; const float *add; int64_t ldadd;
  float alpha = 1.f;
};

// the pairs of planes that a product needs, smallest first: of terms of 8 bits each, those that reach 24 bits
int plane_pairs(int na, int nb, uint32_t &pa, uint32_t &pb) {
  int n = 0;
  const int most = std::max(na, nb) - 1;
  pa = pb = 0;
  for (int sum = most; sum >= 0; --sum)
    for (int a = std::min(sum, na - 1); a >= 0 && sum - a < nb; --a) { pa |= (uint32_t)a << (4 * n); pb |= (uint32_t)(sum - a) << (4 * n); ++n; }
  return n;
}

// How a product is cut: tiles of 256 or 128 (TI), and splits of the sequence of slabs, whose float32 results a second launch adds up.  The
// shortest by what was measured, in microseconds: a slab takes a tile of 256 alone on its CU 1.7 (with all CUs at work; the clock gives way),
// a tile of 128 0.55 alone (four stages: a slab is asked for three slabs ahead; two stages, 0.8), 1.0 beside a second one (two
// stages each), 0.58 each where they follow one another; 4 ... 11 for a tile's start and end; a join 3 and its traffic at 4 TB/s.
// Against all cuts of 19 shapes between 256 x 256 x 512 and 8192 x 2048 x 8192 the choice is within 15 % of the best.  For example
// 2000 x 1000 x 50000: 186 (256, 8 splits), 206 (128, 4), 637 (128, 1); 2048 x 2048 x 2048: 21 (128, 1; two stages 29), 41 (128, 2),
// 47 (256, 1); 256 x 256 x 4096: 11 (128, 16), 26 (128, 1).
// tile_end: what a tile of 128 has to do behind its products beyond a plain store.
// tail: splits of the last round's tiles, where the others fill the GPU a whole number of times and these leave much of it idle for as long
// again: 1000 x 50001 x 1999 with three planes a side, 784 tiles of 256 in four rounds, 665 us; in three and the 16 left over in
// 16 splits each, 602 with their join.
struct GemmCut { int ti, splits, per_split; size_t bytes; int stages, tail; double us; };
constexpr int64_t CUS = 256, BIG_TILE = 256;
constexpr int SPLITS[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64, 96, 128, 192, 256, 384, 512};
inline double join_us(int64_t M, int64_t N, int splits) { return splits > 1 ? 3.0 + (double)splits * (double)M * (double)N * 2e-6 : 0.0; }
inline size_t part_bytes(int64_t M, int64_t N, int splits) { return splits > 1 ? align_up((size_t)splits * M * round_up(N, 8) * sizeof(float)) : 0; }
GemmCut gemm_cut(int64_t M, int64_t N, int64_t K, int planes_a, int planes_b, int most = 512, double tile_end = 0.0) {
  uint32_t unused_a, unused_b;
  const int64_t all = (K + TG_BK - 1) / TG_BK * plane_pairs(planes_a, planes_b, unused_a, unused_b);
  GemmCut best = {2, 1, (int)all, 0, 2, 1, INFINITY};
  const int64_t big = ((M + BIG_TILE - 1) / BIG_TILE) * ((N + BIG_TILE - 1) / BIG_TILE), rest = big % CUS;
  int tail = 1;
  double saved = 0.0;
  if (big > CUS && rest > 0 && most > LOGIT_SPLITS) {
    tail = (int)std::max<int64_t>(1, std::min(CUS / rest, all / 2));
    saved = 6.0 + 1.7 * (double)all - (8.0 + 1.7 * (double)((all + tail - 1) / tail) + 3.0 + (double)(rest * tail) * 0.13);
    if (tail < 2 || saved < 5.0) { tail = 1; saved = 0.0; }
  }
  for (int ti : {2, 4})
    for (int splits : SPLITS) {
      if (splits > 1 && (splits > all / 2 || splits > most)) break;
      const int64_t tile = 64 * ti, tiles = ((M + tile - 1) / tile) * ((N + tile - 1) / tile), per = (all + splits - 1) / splits;
      const double each = (double)((tiles * splits + 255) / 256);       // workgroups per CU
      double us = ti == 4 ? 5.0 + each * (6.0 + 1.7 * (double)per) : 4.0 + (double)per * (each <= 1.0 ? 0.55 : each <= 2.0 ? 1.0 : 0.58 * each) + tile_end * each;
      us += join_us(M, N, splits);
      const bool with_tail = ti == 4 && splits == 1 && tail > 1;
      if (with_tail) us -= saved;
      if (us < best.us) best = {ti, (int)((all + per - 1) / per), (int)per, 0, ti == 2 && each <= 1.0 ? 4 : 2, with_tail ? tail : 1, us};
    }
  best.bytes = part_bytes(M, N, best.splits);
  if (best.tail > 1) best.bytes = align_up((size_t)best.tail * rest * BIG_TILE * BIG_TILE * sizeof(float));
  return best;
}
template <int TI, int STAGES, int END> void gemm_launch(const TrainGemmArgs &g, int alie, int blie, hipStream_t s) {
  const int64_t total = (int64_t)g.tiles * g.splits;
  const dim3 grid((unsigned)((total + 7) / 8 * 8));
  if (alie == LIE_K && blie == LIE_K) train_gemm_kernel<TI, STAGES, LIE_K, LIE_K, END><<<grid, 256, 0, s>>>(g);
  else if (alie == LIE_K) train_gemm_kernel<TI, STAGES, LIE_K, LIE_ROWS, END><<<grid, 256, 0, s>>>(g);
  else if constexpr (END == END_PLAIN) train_gemm_kernel<TI, STAGES, LIE_ROWS, LIE_ROWS, END><<<grid, 256, 0, s>>>(g);
}
template <int END> void gemm_launch(const TrainGemmArgs &g, const GemmCut &cut, int alie, int blie, hipStream_t s) {
  if (cut.ti == 4) gemm_launch<4, 2, END>(g, alie, blie, s);
  else if (cut.stages == 4) gemm_launch<2, 4, END>(g, alie, blie, s);
  else gemm_launch<2, 2, END>(g, alie, blie, s);
}
void gemm_args(const Operand &a, const Operand &b, int64_t M, int64_t N, int64_t K, const GemmCut &cut, TrainGemmArgs &g) {
  g = {};
  g.a = a.p; g.b = b.p; g.lda = a.ld; g.ldb = b.ld; g.a_plane = a.plane; g.b_plane = b.plane;
  g.M = (int32_t)M; g.N = (int32_t)N; g.K = (int32_t)K;
  g.products = plane_pairs(a.planes, b.planes, g.plane_a, g.plane_b);
  g.tiles_m = (int32_t)((M + 64 * cut.ti - 1) / (64 * cut.ti)); g.tiles_n = (int32_t)((N + 64 * cut.ti - 1) / (64 * cut.ti));
  g.splits = cut.splits; g.per_split = cut.per_split;
  g.tiles = g.tiles_m * g.tiles_n;
  g.padded = (a.padded ? 1 : 0) | (b.padded ? 2 : 0);
  g.alpha = 1.f;
}
// where C goes: with several splits their results lie one behind the other in `part`
void gemm_result(TrainGemmArgs &g, const Result &c, float *part) {
  if (g.splits > 1) { g.c = part; g.ldc = round_up(g.N, 8); g.c_split = g.M * g.ldc; g.store = STORE_F32; }
  else { g.c = c.c; g.ldc = c.ldc; g.add = c.add; g.ldadd = c.ldadd; g.store = c.store; g.alpha = c.alpha; }
}
// sums: go along, and are struck out there
int gemm_join(const TrainGemmArgs &g, const Result &c, RowSums &sums, hipStream_t s) {
  JoinArgs j = {};
  j.part = static_cast<const float *>(g.c); j.stride = g.c_split; j.splits = g.splits; j.c = c.c; j.ldc = c.ldc; j.add = c.add; j.ldadd = c.ldadd;
  j.alpha = c.alpha; j.cols = g.N; j.pitch = (int32_t)g.ldc; j.store = c.store; j.per_row = (uint32_t)(g.ldc / 8);
  return by_rows(g.M, j.per_row, [&](int64_t r, uint32_t pieces, dim3 grid) {
    j.row0 = r; j.pieces = pieces;
    const bool eight = g.splits >= 16 && pieces < (1u << 24);
    j.blocks = eight ? (pieces + 31) / 32 : grid.x;
    j.sums = sums;
    sums.out = nullptr;
    const dim3 all(j.blocks + (j.sums.out ? (j.sums.cols + 15) / 16 : 0));
    if (eight) train_join_kernel<8><<<all, 256, 0, s>>>(j); else train_join_kernel<1><<<all, 256, 0, s>>>(j);
  });
}
// C = A B^T; `part`: scratch of gemm_cut's size
int gemm(const Operand &a, const Operand &b, int64_t M, int64_t N, int64_t K, const Result &c, float *part, RowSums &sums, hipStream_t s) {
  const GemmCut cut = gemm_cut(M, N, K, a.planes, b.planes);
  TrainGemmArgs g;
  gemm_args(a, b, M, N, K, cut, g);
  gemm_result(g, c, part);
  if (cut.splits == 1) {
    const int32_t all = g.per_split, rest = cut.tail > 1 ? (int32_t)(g.tiles % CUS) : 0;
    g.tiles -= rest;
    gemm_launch<END_PLAIN>(g, cut, a.lie, b.lie, s);
    HIP_TRY(hipGetLastError());
    if (rest == 0) return SHAMPOO_OK;
    g.tile0 = g.tiles; g.tiles = rest; g.by_tile = 1;
    g.per_split = (all + cut.tail - 1) / cut.tail; g.splits = (all + g.per_split - 1) / g.per_split;
    g.c = part; g.ldc = BIG_TILE; g.c_split = rest * BIG_TILE * BIG_TILE; g.add = nullptr; g.alpha = 1.f; g.store = STORE_F32;
    gemm_launch<END_PLAIN>(g, cut, a.lie, b.lie, s);
    HIP_TRY(hipGetLastError());
    const JoinTilesArgs j = {part, g.c_split, g.splits, c.c, c.ldc, c.add, c.ldadd, g.M, g.N, g.tiles_m, g.tiles_n, g.tile0, (int32_t)BIG_TILE, c.store, c.alpha};
    train_join_tiles_kernel<<<dim3((unsigned)(rest * (BIG_TILE * BIG_TILE / 8 / 256))), 256, 0, s>>>(j);
    HIP_TRY(hipGetLastError());
    return SHAMPOO_OK;
  }
  gemm_launch<END_PLAIN>(g, cut, a.lie, b.lie, s);
  HIP_TRY(hipGetLastError());
  return gemm_join(g, c, sums, s);
}

// Two products, the second with both operands along rows: in one launch of tiles of 128, four workgroups per CU at most, where that is
// shorter by gemm_cut's model and 2 us for a launch.  The gradients of 256 x 2048 x 1000 in float32: 15 + 18 us, together 21.5; of
// 32 x 256 x 1000 in bf16 5.4 + 6.1, together 6.4; with more than one workgroup per CU the whole of 100 x 1024 x 10000 in bf16
// 45.8, 39.0 together.  Of 18 shapes in both types one was longer together (by 2 %, 700 x 700 x 7000 in float32).
struct PairCut { GemmCut first, second; bool together; size_t bytes; };
struct Product { int64_t M, N, K; int planes_a, planes_b; };
PairCut pair_cut(const Product &f, const Product &g) {
  const GemmCut one = gemm_cut(f.M, f.N, f.K, f.planes_a, f.planes_b), two = gemm_cut(g.M, g.N, g.K, g.planes_a, g.planes_b);
  PairCut best = {one, two, false, std::max(one.bytes, two.bytes)};
  double shortest = one.us + two.us + 2.0;
  uint32_t unused_a, unused_b;
  const auto tiles = [](const Product &p) { return (p.M + 127) / 128 * ((p.N + 127) / 128); };
  const auto slabs = [&](const Product &p) { return (p.K + TG_BK - 1) / TG_BK * plane_pairs(p.planes_a, p.planes_b, unused_a, unused_b); };
  const int64_t tiles_f = tiles(f), tiles_g = tiles(g), all_f = slabs(f), all_g = slabs(g);
  for (int sf : SPLITS) {
    if (tiles_f * sf + tiles_g > 4 * CUS || (sf > 1 && sf > all_f / 2)) break;
    for (int sg : SPLITS) {
      if (tiles_f * sf + tiles_g * sg > 4 * CUS || (sg > 1 && sg > all_g / 2)) break;
      const int64_t per_f = (all_f + sf - 1) / sf, per_g = (all_g + sg - 1) / sg, longest = std::max(per_f, per_g);
      const bool alone = round_up(tiles_f * sf, 8) + round_up(tiles_g * sg, 8) <= CUS;        // on its CU
      const double work = (double)(tiles_f * sf * per_f + tiles_g * sg * per_g) / (double)CUS;
      const double us = 4.0 + (alone ? 0.55 * (double)longest : std::max((double)longest, 0.58 * work)) + join_us(f.M, f.N, sf) + join_us(g.M, g.N, sg);
      if (us < shortest) {
        shortest = us;
        best.first = {2, (int)((all_f + per_f - 1) / per_f), (int)per_f, 0, alone ? 4 : 2, 1, us};
        best.second = {2, (int)((all_g + per_g - 1) / per_g), (int)per_g, 0, best.first.stages, 1, us};
        best.first.bytes = part_bytes(f.M, f.N, best.first.splits); best.second.bytes = part_bytes(g.M, g.N, best.second.splits);
        best.together = true; best.bytes = best.first.bytes + best.second.bytes;
      }
    }
  }
  return best;
}
// C = A B^T and E = D F^T in one launch, cut by pair_cut
int gemm_pair(const Operand &a, const Operand &b, const Product &f, const Result &c, const Operand &d, const Operand &e, const Product &g,
              const Result &r, const PairCut &cut, float *part, RowSums &sums, hipStream_t s) {
  TrainGemmArgs x, y;
  gemm_args(a, b, f.M, f.N, f.K, cut.first, x);
  gemm_args(d, e, g.M, g.N, g.K, cut.second, y);
  gemm_result(x, c, part);
  gemm_result(y, r, part + cut.first.bytes / sizeof(float));
  const int blocks = (int)round_up(x.tiles * x.splits, 8);
  const dim3 grid((unsigned)(blocks + round_up(y.tiles * y.splits, 8)));
  if (cut.first.stages == 4) {
    if (b.lie == LIE_K) train_gemm_pair_kernel<4, LIE_K><<<grid, 256, 0, s>>>(x, y, blocks);
    else train_gemm_pair_kernel<4, LIE_ROWS><<<grid, 256, 0, s>>>(x, y, blocks);
  } else {
    if (b.lie == LIE_K) train_gemm_pair_kernel<2, LIE_K><<<grid, 256, 0, s>>>(x, y, blocks);
    else train_gemm_pair_kernel<2, LIE_ROWS><<<grid, 256, 0, s>>>(x, y, blocks);
  }
  HIP_TRY(hipGetLastError());
  if (x.splits > 1) TRY(gemm_join(x, c, sums, s));
  if (y.splits > 1) TRY(gemm_join(y, r, sums, s));
  return SHAMPOO_OK;
}

// A matrix of the caller as an operand: as it lies, or as planes in scratch (float32; rows that the products cannot read to their
// slabs' end: `along`, 64 where the columns are k in some product, otherwise 8).
struct Source {
  int32_t dtype; int64_t rows, cols, ld; int along;
  bool zeros = false;        // a copy has them behind its last row, to the next multiple of 64
  bool copy() const { return dtype != SHAMPOO_GRAD_BF16 || cols % along != 0 || ld % 8 != 0 || ld > MAX_LD; }
  int planes() const { return dtype == SHAMPOO_GRAD_F32 ? 3 : 1; }
  int64_t ldp() const { return round_up(cols, 64); }
  int64_t held() const { return zeros ? round_up(rows, TG_BK) : rows; }
  uint16_t *take(Arena &a) const { return copy() ? a.take<uint16_t>((size_t)planes() * held() * ldp()) : nullptr; }
  Operand operand(const void *p, const uint16_t *scratch, int lie) const {
    if (!copy()) return {static_cast<const uint16_t *>(p), ld, 0, 1, lie};
    return {scratch, ldp(), held() * ldp(), planes(), lie, zeros};
  }
  PlanesTask task(const void *p, uint16_t *scratch) const {
    PlanesTask t = {};
    t.from = dtype == SHAMPOO_GRAD_F32 ? FROM_F32 : FROM_BF16; t.planes = planes(); t.rows = held();
    t.g.rows = rows; t.g.x = p; t.g.ldx = ld; t.g.out = scratch; t.g.plane = held() * ldp(); t.g.ld = ldp(); t.g.cols = (int32_t)cols;
    return t;
  }
};

// ---------------------------------------------------------------------------
// Cross entropy
// ---------------------------------------------------------------------------
struct CrossEntropyPlan {
  Source x, w;
  int planes = 0;            // of g beside float32 logits (twice: alone); 0: in the place of 16-bit ones
  bool twice = false;        // the logits' product runs a second time and leaves g
  int64_t ldz = 0, spans = 0, piece = 0, pieces = 0, range_rows = 1, ranges = 1;
  bool sum = false;          // bf16 dw of several pieces: summed in scratch
  size_t bytes = 0;
  uint16_t *xp, *wp, *g;
  float *z, *top, *coef, *share, *target_z, *acc, *sums, *part;
  float2 *stats;
  int grad_planes() const { return std::max(planes, 1); }
  // the logits' product over n rows: where it stores float32 ones, 0.4 us more for the end of a tile of 128 (1999 x 1000 x 50001: 354 us
  // in 25 tiles of 128 a CU, 330 in seven rounds of tiles of 256; 512 x 512 x 32000 in float32 dw 159 us in all, 168)
  GemmCut for_logits(const shampoo_cross_entropy &c, int64_t n) const {
    return gemm_cut(n, c.classes, c.features, x.planes(), w.planes(), twice ? 1 : LOGIT_SPLITS, c.gradients && !twice && planes ? 0.4 : 0.0);
  }
  // the gradients' products over n rows
  Product for_dx(const shampoo_cross_entropy &c, int64_t n) const { return {n, c.features, c.classes, x.planes(), w.planes()}; }
  Product for_dw(const shampoo_cross_entropy &c, int64_t n) const {
    if (c.w_layout == SHAMPOO_OUT_IN) return {c.classes, c.features, n, grad_planes(), x.planes()};
    return {c.features, c.classes, n, x.planes(), grad_planes()};
  }
};
int cross_entropy_plan(const shampoo_cross_entropy &c, void *workspace, CrossEntropyPlan &p) {
  if (c.rows < 0 || c.features < 1 || c.classes < 1) return SHAMPOO_ERR_SHAPE;
  if (c.rows > MAX_ROWS || c.features > MAX_FEATURES || c.classes > MAX_OUT) return SHAMPOO_ERR_UNSUPPORTED;
  if (!dtype_ok(c.dtype) || !dtype_ok(c.grad_dtype) || (c.w_layout != SHAMPOO_OUT_IN && c.w_layout != SHAMPOO_IN_OUT)) return SHAMPOO_ERR_HYPER;
  if (c.gradients && c.dtype == SHAMPOO_GRAD_F32 && c.grad_dtype != SHAMPOO_GRAD_F32) return SHAMPOO_ERR_HYPER;
  const bool out_in = c.w_layout == SHAMPOO_OUT_IN;
  const int64_t wcols = out_in ? c.features : c.classes, d = c.features, v = c.classes;
  if (((v + 127) / 128) * ((d + 127) / 128) > MAX_TILES) return SHAMPOO_ERR_UNSUPPORTED;
  if (c.ldx < d || c.ldw < wcols || (c.gradients && (c.lddx < d || c.lddw < wcols))) return SHAMPOO_ERR_SHAPE;
  p.x = {c.dtype, c.rows, d, c.ldx, TG_BK};
  p.w = {c.dtype, out_in ? v : d, wcols, c.ldw, TG_BK};
  // a float32 result needs g to float32 accuracy, and that needs the logits so
  p.planes = c.grad_dtype == SHAMPOO_GRAD_F32 ? 3 : c.has_bias ? 1 : 0;
  // Once more 2 features operations per logit (six times that in float32), or 4 bytes (16-bit logits) or 8 of traffic.  4096 rows, 32000 classes
  // (float32: 8000), us with logits kept / made twice: bf16, bf16 dw: 406 / 384 (128 features), 615 / 625 (384); bf16, float32 dw:
  // 859 / 754 (256), 1078 / 1029 (512), 1479 / 1538 (768); float32: 282 / 239 (64), 345 / 352 (128).
  p.twice = c.gradients && !c.has_bias && d <= (c.dtype == SHAMPOO_GRAD_F32 ? 96 : p.planes ? 640 : 192);
  if (p.twice) p.planes = std::max(p.planes, 1);
  p.ldz = round_up(v, 64);
  p.spans = round_up(v, 256) / 64;
  const size_t per_row = (size_t)p.spans * sizeof(float2) + (c.gradients ? (size_t)p.ldz * (p.twice ? 2 * p.planes : p.planes ? 4 + 2 * p.planes : 2) : 0);
  p.piece = std::min<int64_t>(round_up(std::max<int64_t>(c.rows, 1), PIECE_ROWS),
                              std::min(MAX_PIECE_ROWS, std::max<int64_t>(PIECE_ROWS, (int64_t)(LOGIT_BYTES / per_row) / PIECE_ROWS * PIECE_ROWS)));
  p.pieces = (c.rows + p.piece - 1) / p.piece;
  p.sum = c.gradients && p.pieces > 1 && c.grad_dtype == SHAMPOO_GRAD_BF16;
  // rows of a thread of softmax_grad_kernel: 64 where that leaves a thousand workgroups
  p.range_rows = std::min<int64_t>(64, std::max<int64_t>(1, std::min(p.piece, c.rows) * ((p.ldz + 2047) / 2048) / 1024));
  p.ranges = (p.piece + p.range_rows - 1) / p.range_rows;
  Arena a(workspace);
  p.xp = p.x.take(a); p.wp = p.w.take(a);
  p.top = a.take<float>(p.piece); p.coef = a.take<float>(p.piece); p.share = a.take<float>(p.piece); p.target_z = a.take<float>(p.piece);
  p.stats = a.take<float2>((size_t)p.spans * p.piece);
  if (c.gradients) {
    if (p.planes && !p.twice) p.z = a.take<float>((size_t)p.piece * p.ldz);
    p.g = a.take<uint16_t>((size_t)p.grad_planes() * p.piece * p.ldz);
    if (p.sum) p.acc = a.take<float>((size_t)p.w.rows * p.w.cols);
    if (c.has_bias) p.sums = a.take<float>((size_t)p.ranges * v);
  }
  size_t part = 0;
  for (int64_t n : {p.piece, c.rows - std::max<int64_t>(0, p.pieces - 1) * p.piece, c.rows}) {      // all pieces, the last one, a single one
    if (n < 1 || n > p.piece) continue;
    part = std::max(part, p.for_logits(c, n).bytes);
    if (!c.gradients) continue;
    const Product fx = p.for_dx(c, n), fw = p.for_dw(c, n);
    for (const Product &f : {fx, fw}) part = std::max(part, gemm_cut(f.M, f.N, f.K, f.planes_a, f.planes_b).bytes);
    part = std::max(part, pair_cut(fx, fw).bytes);
  }
  if (part) p.part = a.take<float>(part / sizeof(float));
  p.bytes = a.used;
  return SHAMPOO_OK;
}

// ---------------------------------------------------------------------------
// Weight gradient from a checkpoint
// ---------------------------------------------------------------------------
struct WeightGradPlan {
  Source dy;
  int planes = 1;            // of a(x)
  int64_t ldp = 0, piece = 0, pieces = 0, parts = 1, part_rows = 1;
  bool sum = false;
  size_t bytes = 0;
  uint16_t *xp, *dyp;
  float *acc, *sums, *part;
};
int weight_grad_plan(int64_t rows, int32_t in, int32_t out, int32_t activation, int32_t dtype, int64_t lddy, int32_t grad_dtype, bool bias,
                     void *workspace, WeightGradPlan &p) {
  if (rows < 0 || in < 1 || out < 1 || lddy < out) return SHAMPOO_ERR_SHAPE;
  if (rows > MAX_ROWS || in > MAX_FEATURES || out > MAX_OUT || (((int64_t)in + 127) / 128) * (((int64_t)out + 127) / 128) > MAX_TILES)
    return SHAMPOO_ERR_UNSUPPORTED;
  if (!dtype_ok(dtype) || !dtype_ok(grad_dtype) || activation < ACT_NONE || activation > ACT_SILU) return SHAMPOO_ERR_HYPER;
  if (dtype == SHAMPOO_GRAD_F32 && grad_dtype != SHAMPOO_GRAD_F32) return SHAMPOO_ERR_HYPER;
  p.dy = {dtype, rows, out, lddy, 8, true};
  // a code times its scale is a bf16 value, and so is its ReLU; other activations take three planes for a float32 result
  p.planes = activation == ACT_NONE || activation == ACT_RELU || grad_dtype != SHAMPOO_GRAD_F32 ? 1 : 3;
  p.ldp = round_up(in, 64);
  p.piece = std::min<int64_t>(round_up(std::max<int64_t>(rows, 1), PIECE_ROWS),
                              std::max<int64_t>(PIECE_ROWS, (int64_t)(PLANE_BYTES / ((size_t)p.ldp * 2 * p.planes)) / PIECE_ROWS * PIECE_ROWS));
  p.pieces = (rows + p.piece - 1) / p.piece;
  p.sum = p.pieces > 1 && grad_dtype == SHAMPOO_GRAD_BF16;
  // parts of the rows for the column sums: 256, fewer where those were more than 2^22 workgroups of 64 columns
  const int64_t most = std::min<int64_t>(256, MAX_SUM_BLOCKS / (((int64_t)out + 63) / 64));
  p.part_rows = rows <= 128 ? 128 : std::max<int64_t>(64, (rows + most - 1) / most);
  p.parts = std::max<int64_t>(1, (rows + p.part_rows - 1) / p.part_rows);
  Arena a(workspace);
  p.xp = a.take<uint16_t>((size_t)p.planes * p.piece * p.ldp);
  p.dyp = p.dy.take(a);
  if (p.sum) p.acc = a.take<float>((size_t)in * out);
  if (bias && p.parts > 1) p.sums = a.take<float>((size_t)p.parts * out);
  size_t part = 0;
  for (int64_t n : {p.piece, rows - std::max<int64_t>(0, p.pieces - 1) * p.piece, rows}) {
    if (n < 1 || n > p.piece) continue;
    part = std::max(part, std::max(gemm_cut(out, in, n, p.dy.planes(), p.planes).bytes, gemm_cut(in, out, n, p.planes, p.dy.planes()).bytes));
  }
  if (part) p.part = a.take<float>(part / sizeof(float));
  p.bytes = a.used;
  return SHAMPOO_OK;
}

// where the sum over pieces of a weight gradient goes: float32 ones add up in place, bf16 ones in scratch until the last
Result piece_result(void *dw, int64_t lddw, int32_t grad_dtype, float *acc, int64_t cols, bool first, bool last) {
  if (grad_dtype == SHAMPOO_GRAD_F32) return {dw, lddw, STORE_F32, first ? nullptr : static_cast<const float *>(dw), lddw};
  if (last) return {dw, lddw, STORE_BF16, first ? nullptr : acc, cols};
  return {acc, cols, STORE_F32, first ? nullptr : acc, cols};
}

// ---------------------------------------------------------------------------
// Residual norm
// ---------------------------------------------------------------------------
// Teams of the backward pass: what the GPU holds at a time (two or three wavefronts per SIMD by registers; 512 threads: one team per CU),
// and at least four rows each, since every team leaves a row of sums.
inline int norm_threads(int32_t cols) { return cols <= 512 ? 64 : cols <= 1024 ? 128 : cols <= 2048 ? 256 : 512; }
inline int64_t norm_teams(const shampoo_residual_norm &c) {
  const int64_t held = c.cols <= 2048 ? 3 * 256 * 256 / norm_threads(c.cols) : 256;
  return std::max<int64_t>(1, std::min(held, c.rows / 4));
}
int residual_norm_ok(const shampoo_residual_norm &c) {
  if (c.rows < 0 || c.cols < 1 || c.gates < 0) return SHAMPOO_ERR_SHAPE;
  if (c.rows > MAX_ROWS || c.cols > MAX_NORM_COLS) return SHAMPOO_ERR_UNSUPPORTED;
  if (c.gates > 0 && c.rows % c.gates != 0) return SHAMPOO_ERR_SHAPE;
  if (!dtype_ok(c.dtype) || c.post < NORM_NONE || c.post > NORM_LAYER || c.pre < NORM_NONE || c.pre > NORM_LAYER) return SHAMPOO_ERR_HYPER;
  if (!(c.epsilon >= 0.f) || !std::isfinite(c.epsilon) || !std::isfinite(c.scale)) return SHAMPOO_ERR_HYPER;
  if ((c.post != NORM_NONE && !c.w_post) || (c.pre != NORM_NONE && !c.w_pre) || (c.gates > 0 && !c.gate)) return SHAMPOO_ERR_NULL;
  return SHAMPOO_OK;
}
ResidualNormArgs residual_norm_args(const shampoo_residual_norm &c) {
  ResidualNormArgs g = {};
  g.w_post = c.w_post; g.b_post = c.post == NORM_LAYER ? c.b_post : nullptr;
  g.w_pre = c.w_pre; g.b_pre = c.pre == NORM_LAYER ? c.b_pre : nullptr;
  g.gate = c.gates > 0 ? c.gate : nullptr;
  g.rows = c.rows; g.cols = c.cols; g.post = c.post; g.pre = c.pre; g.epsilon = c.epsilon; g.alpha = c.scale;
  g.group_rows = c.gates > 0 ? c.rows / c.gates : c.rows;
  return g;
}
struct NormChunks { int64_t rows, chunks; int32_t per_group; };
// A team of the backward pass has rows of one group, or several whole groups where there are more than teams.
NormChunks norm_chunks(const shampoo_residual_norm &c) {
  const int64_t groups = std::max<int64_t>(1, c.gates), group_rows = c.rows / groups;
  const int64_t teams = norm_teams(c);
  if (groups >= teams) {
    const int64_t each = (groups + teams - 1) / teams;
    return {each * group_rows, (groups + each - 1) / each, 0};
  }
  const int64_t want = std::max<int64_t>(1, std::min(teams / groups, group_rows));
  const int64_t rows = std::max<int64_t>(1, (group_rows + want - 1) / want), per = std::max<int64_t>(1, (group_rows + rows - 1) / rows);
  return {rows, per * groups, (int32_t)per};
}

// Threads and pieces of eight features per thread for a row (residual_norm.h)
template <typename F> void norm_forward_variant(int32_t cols, F &&launch) {
#define VARIANT(TPR, NJ) launch(std::integral_constant<int, TPR>(), std::integral_constant<int, NJ>())
  if (cols <= 512) VARIANT(64, 1);
  else if (cols <= 1024) VARIANT(64, 2);
  else if (cols <= 2048) VARIANT(64, 4);
  else if (cols <= 4096) VARIANT(256, 2);
  else if (cols <= 8192) VARIANT(256, 4);
  else VARIANT(512, 4);
}
template <typename F> void norm_backward_variant(int32_t cols, F &&launch) {
  if (cols <= 512) VARIANT(64, 1);
  else if (cols <= 1024) VARIANT(128, 1);
  else if (cols <= 2048) VARIANT(256, 1);
  else if (cols <= 4096) VARIANT(512, 1);
  else if (cols <= 8192) VARIANT(512, 2);
  else VARIANT(512, 4);
#undef VARIANT
}
// at most 2^22 workgroups in a launch, whose threads have 32 bits
template <typename T> int launch_norm_forward(ResidualNormArgs g, hipStream_t s) {
  int rc = SHAMPOO_OK;
  norm_forward_variant(g.cols, [&](auto tpr, auto nj) {
    constexpr int TPR = decltype(tpr)::value;
    constexpr int64_t TEAMS = TPR > 256 ? 1 : 256 / TPR, AT_ONCE = TEAMS << 22;
    for (; g.row0 < g.rows && rc == SHAMPOO_OK; g.row0 += AT_ONCE) {
      const int64_t rows = std::min(AT_ONCE, g.rows - g.row0);
      residual_norm_forward_kernel<T, TPR, decltype(nj)::value><<<dim3((unsigned)((rows + TEAMS - 1) / TEAMS)), TEAMS * TPR, 0, s>>>(g);
      if (hipGetLastError() != hipSuccess) rc = SHAMPOO_ERR_HIP;
    }
  });
  return rc;
}
template <typename T> int launch_norm_backward(const ResidualNormArgs &g, bool bias, hipStream_t s) {
  norm_backward_variant(g.cols, [&](auto tpr, auto nj) {
    constexpr int TPR = decltype(tpr)::value, NJ = decltype(nj)::value, TEAMS = TPR == 64 ? 4 : 1;
    const dim3 grid((unsigned)((g.teams + TEAMS - 1) / TEAMS));
    if (bias) residual_norm_backward_kernel<T, TPR, NJ, true><<<grid, TEAMS * TPR, 0, s>>>(g);
    else residual_norm_backward_kernel<T, TPR, NJ, false><<<grid, TEAMS * TPR, 0, s>>>(g);
  });
  HIP_TRY(hipGetLastError());
  return SHAMPOO_OK;
}

int checkpoint_ok(int64_t rows, int32_t cols, const void *packed, size_t bytes) {
  if (rows < 0 || cols < 1) return SHAMPOO_ERR_SHAPE;
  if (rows > MAX_ROWS || cols > MAX_PACKED_COLS) return SHAMPOO_ERR_UNSUPPORTED;
  return workspace_ok(packed, bytes, shampoo_checkpoint_bytes(rows, cols));
}

}  // namespace

// ---------------------------------------------------------------------------
// extern "C" boundary
// ---------------------------------------------------------------------------
extern "C" {

size_t shampoo_linear_cross_entropy_workspace_bytes(const shampoo_cross_entropy *c) {
  CrossEntropyPlan p;
  return c && cross_entropy_plan(*c, nullptr, p) == SHAMPOO_OK ? p.bytes : 0;
}

int shampoo_linear_cross_entropy(const shampoo_cross_entropy *c, const void *x, const void *w, const float *bias, const int64_t *targets,
                                 const float *weight, float scale, float *loss, void *dx, void *dw, float *dbias, void *workspace,
                                 size_t workspace_bytes, void *stream) {
  if (!c) return SHAMPOO_ERR_NULL;
  CrossEntropyPlan p;
  TRY(cross_entropy_plan(*c, workspace, p));
  if (!w || (c->rows > 0 && (!x || !targets || !loss)) || (c->has_bias && !bias)) return SHAMPOO_ERR_NULL;
  if (!std::isfinite(scale)) return SHAMPOO_ERR_HYPER;
  if (!aligned(x, 16) || !aligned(w, 16)) return SHAMPOO_ERR_UNSUPPORTED;
  TRY(workspace_ok(workspace, workspace_bytes, p.bytes));
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int64_t d = c->features, v = c->classes;
  const bool out_in = c->w_layout == SHAMPOO_OUT_IN;
  if (!c->gradients) { dx = dw = nullptr; dbias = nullptr; }
  if (!c->has_bias) { bias = nullptr; dbias = nullptr; }
  if (c->rows == 0) {
    if (dw) TRY(launch_zero(dw, p.w.rows, p.w.cols, c->lddw, size_of(c->grad_dtype), s));
    if (dbias) TRY(launch_zero(dbias, 1, v, v, 4, s));
    return SHAMPOO_OK;
  }
  const Operand xo = p.x.operand(x, p.xp, LIE_K), wo = p.w.operand(w, p.wp, out_in ? LIE_K : LIE_ROWS);
  if (p.x.copy() && p.w.copy()) TRY(launch_planes(p.x.task(x, p.xp), p.w.task(w, p.wp), s));
  else if (p.x.copy()) TRY(launch_planes(p.x.task(x, p.xp), s));
  else if (p.w.copy()) TRY(launch_planes(p.w.task(w, p.wp), s));
  // scale = power alpha, alpha in [1, 2); very small ones as they are
  const float power = std::fabs(scale) < 0x1p-100f ? scale : std::copysign(std::ldexp(1.f, std::ilogb(scale)), scale);
  const float alpha = std::fabs(scale) < 0x1p-100f ? 1.f : scale / power;
  for (int64_t k = 0; k < p.pieces; ++k) {
    const int64_t i0 = k * p.piece, n = std::min(p.piece, c->rows - i0);
    Operand xk = xo;
    xk.p += i0 * xo.ld;
    const GemmCut cut = p.for_logits(*c, n);
    const int32_t span = cut.splits > 1 ? 64 : 32 * cut.ti;
    const int store = !c->gradients || p.twice ? STORE_NOTHING : STORE_F32, end = store == STORE_NOTHING || p.planes ? END_LOGITS : END_LOGITS_U16;
    void *const logits = p.planes ? static_cast<void *>(p.z) : p.g;
    TrainGemmArgs z;
    gemm_args(xk, wo, n, v, d, cut, z);
    if (cut.splits > 1) {
      gemm_result(z, {}, p.part);
      gemm_launch<END_PLAIN>(z, cut, xk.lie, wo.lie, s);
      HIP_TRY(hipGetLastError());
      LogitsJoinArgs j = {p.part, z.c_split, z.ldc, cut.splits, logits, p.ldz, end, store, bias, targets + i0, p.stats, p.piece, p.target_z,
                          (int32_t)n, (int32_t)v, (uint32_t)(n * (p.ldz / 8)), (uint32_t)(p.ldz / 8)};
      logits_join_kernel<<<dim3((j.pieces + 63) / 64), 256, 0, s>>>(j);
    } else {
      z.c = logits; z.ldc = p.ldz; z.store = store;
      z.bias = bias; z.targets = targets + i0; z.stats = p.stats; z.stats_ld = p.piece; z.target_z = p.target_z;
      if (end == END_LOGITS_U16) gemm_launch<END_LOGITS_U16>(z, cut, xk.lie, wo.lie, s); else gemm_launch<END_LOGITS>(z, cut, xk.lie, wo.lie, s);
    }
    HIP_TRY(hipGetLastError());
    const RowLossArgs r = {p.stats, p.piece, p.target_z, targets + i0, weight ? weight + i0 : nullptr, power, p.top, p.coef, p.share, loss + i0,
                           (int32_t)n, (int32_t)v, (int32_t)((v + span - 1) / span)};
    const dim3 grid((unsigned)((p.ldz / 8 + 255) / 256), (unsigned)((round_up(n, TG_BK) + p.range_rows - 1) / p.range_rows));   // zeros behind the last row
    RowSums sums = {p.sums, dbias, (int32_t)grid.y, (int32_t)v, k > 0};      // later pieces add to dbias
    const bool wanted = dx || dw || dbias;
    if (!wanted || p.twice || grid.x > 1) {                   // otherwise softmax_grad_kernel ends the rows
      row_loss_kernel<<<dim3((unsigned)((n + 15) / 16)), 1024, 0, s>>>(r);
      HIP_TRY(hipGetLastError());
    }
    if (!wanted) continue;
    if (p.twice) {
      z.c = p.g; z.top = p.top; z.coef = p.coef; z.share = p.share; z.c_plane = p.piece * p.ldz; z.c_planes = p.planes;
      gemm_launch<END_GRAD>(z, cut, xk.lie, wo.lie, s);
    } else {
      const SoftmaxGradArgs q = {r, p.z, p.ldz, span, p.g, p.piece * p.ldz, dbias ? p.sums : nullptr, (int32_t)p.range_rows, alpha};
      switch (p.planes) {
        case 0: softmax_grad_kernel<0><<<grid, 256, 0, s>>>(q); break;
        case 1: softmax_grad_kernel<1><<<grid, 256, 0, s>>>(q); break;
        default: softmax_grad_kernel<3><<<grid, 256, 0, s>>>(q);
      }
    }
    HIP_TRY(hipGetLastError());
    // dx = g w, dw = g^T x (or its transpose)
    const Operand go = {p.g, p.ldz, p.piece * p.ldz, p.x.planes(), LIE_K}, gt = {p.g, p.ldz, p.piece * p.ldz, p.grad_planes(), LIE_ROWS, true};
    Operand wt = wo;
    wt.lie = out_in ? LIE_ROWS : LIE_K;
    xk.lie = LIE_ROWS;
    const Operand &left = out_in ? gt : xk, &right = out_in ? xk : gt;
    const Product fx = p.for_dx(*c, n), fw = p.for_dw(*c, n);
    const Result to_dx = {!dx ? nullptr : static_cast<char *>(dx) + i0 * c->lddx * size_of(c->dtype), c->lddx, c->dtype == SHAMPOO_GRAD_F32 ? STORE_F32 : STORE_BF16, nullptr, 0, alpha};
    Result to_dw = piece_result(dw, c->lddw, c->grad_dtype, p.acc, p.w.cols, k == 0, k == p.pieces - 1);
    to_dw.alpha = alpha;
    const PairCut pair = dx && dw ? pair_cut(fx, fw) : PairCut();
    if (pair.together) {
      TRY(gemm_pair(go, wt, fx, to_dx, left, right, fw, to_dw, pair, p.part, sums, s));
    } else {
      if (dx) TRY(gemm(go, wt, n, d, v, to_dx, p.part, sums, s));
      if (dw) TRY(gemm(left, right, fw.M, fw.N, fw.K, to_dw, p.part, sums, s));
    }
    TRY(launch_row_sums(sums, s));
  }
  return SHAMPOO_OK;
}

size_t shampoo_checkpoint_bytes(int64_t rows, int32_t cols) {
  if (rows < 0 || rows > MAX_ROWS || cols < 1 || cols > MAX_PACKED_COLS) return 0;
  const size_t pitch = (size_t)round_up(cols, 32);
  return align_up((size_t)rows * pitch) + align_up((size_t)rows * (pitch / 32));
}

int shampoo_checkpoint_pack(const void *x, int32_t dtype, int64_t rows, int32_t cols, int64_t ldx, void *packed, size_t packed_bytes,
                            void *stream) {
  if (rows > 0 && (!x || !packed)) return SHAMPOO_ERR_NULL;
  if (!dtype_ok(dtype)) return SHAMPOO_ERR_HYPER;
  TRY(checkpoint_ok(rows, cols, packed, packed_bytes));
  if (ldx < cols) return SHAMPOO_ERR_SHAPE;
  hipStream_t s = static_cast<hipStream_t>(stream);
  PackArgs g = {};
  g.x = x; g.ldx = ldx; g.p = packed_view(packed, rows, cols);
  g.per_row = (uint32_t)g.p.pitch / 8;
  return by_rows(rows, g.per_row, [&](int64_t r, uint32_t pieces, dim3 grid) {
    g.row0 = r; g.pieces = pieces;
    if (dtype == SHAMPOO_GRAD_F32) checkpoint_pack_kernel<float><<<grid, 256, 0, s>>>(g);
    else checkpoint_pack_kernel<uint16_t><<<grid, 256, 0, s>>>(g);
  });
}

int shampoo_checkpoint_unpack(const void *packed, size_t packed_bytes, int64_t rows, int32_t cols, int32_t activation, void *y, int32_t dtype,
                              int64_t ldy, void *stream) {
  if (rows > 0 && (!packed || !y)) return SHAMPOO_ERR_NULL;
  if (!dtype_ok(dtype) || activation < ACT_NONE || activation > ACT_SILU) return SHAMPOO_ERR_HYPER;
  TRY(checkpoint_ok(rows, cols, packed, packed_bytes));
  if (ldy < cols) return SHAMPOO_ERR_SHAPE;
  hipStream_t s = static_cast<hipStream_t>(stream);
  UnpackArgs g = {};
  g.p = packed_view(packed, rows, cols); g.y = y; g.ldy = ldy; g.activation = activation;
  g.per_row = (uint32_t)g.p.pitch / 8;
  return by_rows(rows, g.per_row, [&](int64_t r, uint32_t pieces, dim3 grid) {
    g.row0 = r; g.pieces = pieces;
    if (dtype == SHAMPOO_GRAD_F32) checkpoint_unpack_kernel<float, false><<<grid, 256, 0, s>>>(g);
    else checkpoint_unpack_kernel<uint16_t, false><<<grid, 256, 0, s>>>(g);
  });
}

int shampoo_checkpoint_activation_grad(const void *packed, size_t packed_bytes, int64_t rows, int32_t cols, int32_t activation, const void *dy,
                                       int32_t dtype, int64_t lddy, void *dx, int64_t lddx, void *stream) {
  if (rows > 0 && (!packed || !dy || !dx)) return SHAMPOO_ERR_NULL;
  if (!dtype_ok(dtype) || activation < ACT_NONE || activation > ACT_SILU) return SHAMPOO_ERR_HYPER;
  TRY(checkpoint_ok(rows, cols, packed, packed_bytes));
  if (lddy < cols || lddx < cols) return SHAMPOO_ERR_SHAPE;
  hipStream_t s = static_cast<hipStream_t>(stream);
  UnpackArgs g = {};
  g.p = packed_view(packed, rows, cols); g.dy = dy; g.lddy = lddy; g.y = dx; g.ldy = lddx; g.activation = activation;
  g.per_row = (uint32_t)g.p.pitch / 8;
  return by_rows(rows, g.per_row, [&](int64_t r, uint32_t pieces, dim3 grid) {
    g.row0 = r; g.pieces = pieces;
    if (dtype == SHAMPOO_GRAD_F32) checkpoint_unpack_kernel<float, true><<<grid, 256, 0, s>>>(g);
    else checkpoint_unpack_kernel<uint16_t, true><<<grid, 256, 0, s>>>(g);
  });
}

size_t shampoo_checkpoint_weight_grad_workspace_bytes(int64_t rows, int32_t in, int32_t out, int32_t activation, int32_t dtype, int64_t lddy,
                                                      int32_t grad_dtype, int32_t want_bias) {
  WeightGradPlan p;
  return weight_grad_plan(rows, in, out, activation, dtype, lddy, grad_dtype, want_bias != 0, nullptr, p) == SHAMPOO_OK ? p.bytes : 0;
}

int shampoo_checkpoint_weight_grad(const void *packed, size_t packed_bytes, int64_t rows, int32_t in, int32_t activation, const void *dy,
                                   int32_t dtype, int32_t out, int64_t lddy, void *dw, int32_t grad_dtype, int32_t w_layout, int64_t lddw,
                                   float *db, void *workspace, size_t workspace_bytes, void *stream) {
  if ((rows > 0 && (!packed || !dy)) || !dw) return SHAMPOO_ERR_NULL;
  WeightGradPlan p;
  TRY(weight_grad_plan(rows, in, out, activation, dtype, lddy, grad_dtype, db != nullptr, workspace, p));
  if (w_layout != SHAMPOO_OUT_IN && w_layout != SHAMPOO_IN_OUT) return SHAMPOO_ERR_HYPER;
  const bool out_in = w_layout == SHAMPOO_OUT_IN;
  if (lddw < (out_in ? in : out)) return SHAMPOO_ERR_SHAPE;
  if (!aligned(dy, 16)) return SHAMPOO_ERR_UNSUPPORTED;
  TRY(checkpoint_ok(rows, in, packed, packed_bytes));
  TRY(workspace_ok(workspace, workspace_bytes, p.bytes));
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (rows == 0) {
    TRY(launch_zero(dw, out_in ? out : in, out_in ? in : out, lddw, size_of(grad_dtype), s));
    if (db) TRY(launch_zero(db, 1, out, out, 4, s));
    return SHAMPOO_OK;
  }
  ColumnSums columns = {};
  RowSums sums = {};
  if (db) columns = {{dy, lddy, rows, p.part_rows, p.parts > 1 ? p.sums : db, out, dtype == SHAMPOO_GRAD_BF16}, p.parts};
  if (db && p.parts > 1) sums = {p.sums, db, (int32_t)p.parts, out, 0};
  const Operand dyo = p.dy.operand(dy, p.dyp, LIE_ROWS);
  const bool both = p.dy.copy() && p.pieces == 1;
  if (p.dy.copy() && !both) TRY(launch_planes(p.dy.task(dy, p.dyp), s));
  PlanesTask t = {};
  t.from = FROM_PACKED; t.planes = p.planes;
  t.g.out = p.xp; t.g.ld = p.ldp; t.g.plane = p.piece * p.ldp; t.g.cols = in; t.g.activation = activation;
  for (int64_t k = 0; k < p.pieces; ++k) {
    const int64_t i0 = k * p.piece, n = std::min(p.piece, rows - i0);
    const Operand xo = {p.xp, p.ldp, p.piece * p.ldp, p.planes, LIE_ROWS, true};
    Operand dk = dyo;
    dk.p += i0 * dyo.ld;
    t.g.p = packed_view(packed, rows, in);
    t.g.p.codes += i0 * t.g.p.pitch; t.g.p.exps += i0 * (t.g.p.pitch / 32);
    t.g.rows = n; t.rows = round_up(n, TG_BK);              // zeros behind the last row
    if (both) TRY(launch_planes(t, p.dy.task(dy, p.dyp), s, columns)); else TRY(launch_planes(t, s, columns));
    columns.parts = 0;
    const Result r = piece_result(dw, lddw, grad_dtype, p.acc, out_in ? in : out, k == 0, k == p.pieces - 1);
    TRY(out_in ? gemm(dk, xo, out, in, n, r, p.part, sums, s) : gemm(xo, dk, in, out, n, r, p.part, sums, s));
  }
  return launch_row_sums(sums, s);
}

int shampoo_residual_norm_forward(const shampoo_residual_norm *c, const void *r, int64_t ldr, const void *f, int64_t ldf, void *r_out,
                                  int64_t ld_r_out, void *h, int64_t ldh, void *packed_r, void *packed_f, size_t packed_bytes, void *stream) {
  if (!c) return SHAMPOO_ERR_NULL;
  TRY(residual_norm_ok(*c));
  if (c->rows == 0) return SHAMPOO_OK;
  if (!r || !f || !r_out || (c->pre != NORM_NONE && !h) || !packed_r != !packed_f) return SHAMPOO_ERR_NULL;
  if (ldr < c->cols || ldf < c->cols || ld_r_out < c->cols || (c->pre != NORM_NONE && ldh < c->cols)) return SHAMPOO_ERR_SHAPE;
  if (packed_r) {
    TRY(checkpoint_ok(c->rows, c->cols, packed_r, packed_bytes));
    TRY(checkpoint_ok(c->rows, c->cols, packed_f, packed_bytes));
  }
  ResidualNormArgs g = residual_norm_args(*c);
  g.r = r; g.ldr = ldr; g.f = f; g.ldf = ldf; g.r_out = r_out; g.ld_r_out = ld_r_out; g.h = h; g.ldh = ldh;
  g.r8 = packed_view(packed_r, c->rows, c->cols); g.f8 = packed_view(packed_f, c->rows, c->cols);
  hipStream_t s = static_cast<hipStream_t>(stream);
  return c->dtype == SHAMPOO_GRAD_F32 ? launch_norm_forward<float>(g, s) : launch_norm_forward<uint16_t>(g, s);
}

size_t shampoo_residual_norm_backward_workspace_bytes(const shampoo_residual_norm *c) {
  if (!c || residual_norm_ok(*c) != SHAMPOO_OK) return 0;
  return align_up((size_t)norm_chunks(*c).chunks * SUMS * c->cols * sizeof(float));
}

int shampoo_residual_norm_backward(const shampoo_residual_norm *c, int32_t packed, const void *r, int64_t ldr, const void *f, int64_t ldf,
                                   const void *dr_out, int64_t ld_dr_out, const void *dh, int64_t ld_dh, void *dr, int64_t ld_dr, void *df,
                                   int64_t ld_df, float *dgate, float *dw_post, float *db_post, float *dw_pre, float *db_pre, void *workspace,
                                   size_t workspace_bytes, void *stream) {
  if (!c) return SHAMPOO_ERR_NULL;
  TRY(residual_norm_ok(*c));
  if (c->gates == 0) dgate = nullptr;
  if (c->post == NORM_NONE) dw_post = nullptr;
  if (c->post != NORM_LAYER) db_post = nullptr;
  if (c->pre == NORM_NONE) { dw_pre = nullptr; dh = nullptr; }
  if (c->pre != NORM_LAYER) db_pre = nullptr;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int32_t cols = c->cols;
  if (c->rows == 0) {
    if (dgate) TRY(launch_zero(dgate, c->gates, cols, cols, 4, s));
    for (float *p : {dw_post, db_post, dw_pre, db_pre})
      if (p) TRY(launch_zero(p, 1, cols, cols, 4, s));
    return SHAMPOO_OK;
  }
  if (!r || !f || !dr || !df || (c->pre != NORM_NONE && !dh)) return SHAMPOO_ERR_NULL;
  if ((!packed && (ldr < cols || ldf < cols)) || (dr_out && ld_dr_out < cols) || (dh && ld_dh < cols) || ld_dr < cols || ld_df < cols)
    return SHAMPOO_ERR_SHAPE;
  if (packed && (!aligned(r, ALIGN) || !aligned(f, ALIGN))) return SHAMPOO_ERR_WORKSPACE;
  const NormChunks k = norm_chunks(*c);
  TRY(workspace_ok(workspace, workspace_bytes, shampoo_residual_norm_backward_workspace_bytes(c)));
  ResidualNormArgs g = residual_norm_args(*c);
  g.r = r; g.f = f; g.ldr = ldr; g.ldf = ldf;
  if (packed) { g.r8 = packed_view(r, c->rows, cols); g.f8 = packed_view(f, c->rows, cols); }
  g.dr_out = dr_out; g.ld_dr_out = ld_dr_out; g.dh = dh; g.ld_dh = ld_dh; g.dr = dr; g.ld_dr = ld_dr; g.df = df; g.ld_df = ld_df;
  g.dgate = k.per_group ? nullptr : dgate;
  g.partial = static_cast<float *>(workspace);
  g.chunk_rows = k.rows; g.chunks_per_group = k.per_group; g.teams = k.chunks;
  const bool bias = db_post || db_pre || g.b_post;
  TRY(c->dtype == SHAMPOO_GRAD_F32 ? launch_norm_backward<float>(g, bias, s) : launch_norm_backward<uint16_t>(g, bias, s));
  JoinSumsArgs j = {};
  j.part_stride = SUMS * (int64_t)cols; j.out_stride = cols; j.cols = cols;
  int count = 0;
  auto add = [&](const float *in, float *out, int64_t parts) { j.in[count] = in; j.out[count] = out; j.parts[count++] = (int32_t)parts; };
  float *const sums[SUMS] = {nullptr, dw_post, dw_pre, db_post, db_pre};
  for (int q = 0; q < SUMS; ++q)
    if (sums[q]) add(g.partial + q * cols, sums[q], k.chunks);
  if (dgate && k.per_group) {
    j.output_stride = k.per_group * j.part_stride;
    if (count + c->gates <= JOIN_SUMS) {                   // few gates: in the same launch
      for (int64_t o = 0; o < c->gates; ++o) add(g.partial + o * j.output_stride, dgate + o * cols, k.per_group);
    } else {
      JoinSumsArgs gates = j;
      gates.in[0] = g.partial; gates.out[0] = dgate; gates.parts[0] = k.per_group;
      TRY(launch_join_sums(gates, 1, c->gates, s));
    }
  }
  TRY(launch_join_sums(j, count, 1, s));
  return SHAMPOO_OK;
}

}  // extern "C"
