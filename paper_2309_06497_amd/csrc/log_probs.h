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
#include "group.h"
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

// Sums of a part of a row: sum of 2^x and sum of x 2^x, x from z = m in units of log 2.  m = -infinity: nothing there.
struct SoftSums { float m, s, w; };
// the same about another m, no smaller
__device__ __forceinline__ SoftSums about(const SoftSums t, float m, float c) {
  const float d = fmaxf((t.m - m) * c, LP_NOTHING), f = __builtin_amdgcn_exp2f(d);
  return {m, f * t.s, f * fmaf(d, t.s, t.w)};
}

// Over the lanes of a wavefront, by moves between lanes that need no LDS; the result in all of them.
#define LP_DPP(x, ctrl, old) __builtin_amdgcn_update_dpp(old, x, ctrl, 0xf, 0xf, false)
template <typename F> __device__ __forceinline__ float wave_all(float x, float none, F &&f) {
  const int o = __float_as_int(none);
  x = f(x, __int_as_float(LP_DPP(__float_as_int(x), 0x111, o)));          // from 1, 2, 4, 8 lanes before in a row of 16
  x = f(x, __int_as_float(LP_DPP(__float_as_int(x), 0x112, o)));
  x = f(x, __int_as_float(LP_DPP(__float_as_int(x), 0x114, o)));
  x = f(x, __int_as_float(LP_DPP(__float_as_int(x), 0x118, o)));
  x = f(x, __int_as_float(__builtin_amdgcn_update_dpp(o, __float_as_int(x), 0x142, 0xa, 0xf, false)));   // the last of a row to the next one
  x = f(x, __int_as_float(__builtin_amdgcn_update_dpp(o, __float_as_int(x), 0x143, 0xc, 0xf, false)));   // of the first half to the second
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}
__device__ __forceinline__ float wave_max(float x) { return wave_all(x, -INFINITY, [](float p, float q) { return fmaxf(p, q); }); }
__device__ __forceinline__ float wave_sum(float x) { return wave_all(x, 0.f, [](float p, float q) { return p + q; }); }
__device__ __forceinline__ int wave_scan(int x) {            // of this lane and those before it
  x += LP_DPP(x, 0x111, 0);
  x += LP_DPP(x, 0x112, 0);
  x += LP_DPP(x, 0x114, 0);
  x += LP_DPP(x, 0x118, 0);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
  return x;
}
// how many lanes before this one are in a mask
__device__ __forceinline__ int lanes_before(uint64_t mask) { return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0)); }

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

// The `top` largest of many logits.  First by a table: bins of the distance from the largest one, 64 to each doubling of 1 + that distance in units of log 2, up to 255 units (a row that is
// sure of one token has its others far away).  What reaches bin b holds the `top` largest if `top` values do, since equal ones share a bin and larger ones have
// no higher one.  One pass of LDS atomics where a search for a bound takes a count by all lanes for each of its steps: 20 tokens of 1 x 131072 in 11.7 us, by the
// search alone 2.5 more.
constexpr int LP_CHOSEN = LP_MAX_TOP + LP_MAX_TOP / 2, LP_CANDIDATES = 512;
constexpr int LP_BINS = 512;
constexpr uint32_t LP_BIN_SHIFT = 17, LP_BIN_FIRST = 0x3f800000u >> LP_BIN_SHIFT;      // the upper bits of a float32 are the bin
__device__ __forceinline__ uint32_t bin_bits(float z, float largest, float c) { return __float_as_uint(fmaf(largest - z, c, 1.f)); }
__device__ __forceinline__ int bin_of(float z, float largest, float c) { return (int)min((bin_bits(z, largest, c) >> LP_BIN_SHIFT) - LP_BIN_FIRST, (uint32_t)LP_BINS); }   // LP_BINS: none, and NaN
__device__ __forceinline__ bool within_bin(float z, float largest, float c, int bin) { return bin_bits(z, largest, c) < (uint32_t)(bin + 1 + (int)LP_BIN_FIRST) << LP_BIN_SHIFT; }
// the first bin by which `top` values are there, or LP_BINS: there are not so many, or more than LP_CHOSEN
__device__ __forceinline__ int bin_bound(const int *bins, int top, int lane) {
  const int4 p = reinterpret_cast<const int4 *>(bins)[2 * lane], q = reinterpret_cast<const int4 *>(bins)[2 * lane + 1];
  const int here[8] = {p.x, p.y, p.z, p.w, q.x, q.y, q.z, q.w};
  const int all = ((p.x + p.y) + (p.z + p.w)) + ((q.x + q.y) + (q.z + q.w)), upto = wave_scan(all);
  const uint64_t enough = __ballot(upto >= top);
  if (enough == 0) return LP_BINS;
  int n = upto - all, bin = 8 * lane - 1;
#pragma unroll
  for (int k = 0; k < 8; ++k)
    if (n < top) { n += here[k]; ++bin; }
  const int at = __builtin_ctzll(enough);
  return __builtin_amdgcn_readlane(n, at) <= LP_CHOSEN ? __builtin_amdgcn_readlane(bin, at) : LP_BINS;
}

// Where that does not do (tiny spreads, too many in a bin): a bound that `top` to at_most(top) keys reach, or all, where there are no more.  count(b): how many
// are >= b.  The search goes from `above`, which none reaches, in steps that grow until enough do, and by halves from there.
__device__ __forceinline__ int at_most(int top) { return top + max(16, top / 2); }
template <typename Key, typename Count> __device__ __forceinline__ Key bound_of(Key lowest, Key above, Key step, int least, int most, Count &&count) {
  if (count(lowest) <= most) return lowest;
  Key lo = lowest, hi = above;
  while (hi - lo > 1) {
    const Key mid = step != 0 && hi - lo > step ? hi - step : lo + (hi - lo) / 2;
    const int n = count(mid);
    if (n < least) { hi = mid; step <<= 1; }
    else if (n > most) { lo = mid; step = 0; }
    else return mid;
  }
  return lo;                             // more than `most` equal ones, where keys are values alone
}
// What a workgroup of W wavefronts needs for both
template <int W> struct Selection {
  alignas(16) int bins[LP_BINS];
  uint64_t counts[2][W];
  int n_chosen, n_candidates, chosen[LP_CHOSEN];
  uint64_t candidate[LP_CANDIDATES], last[LP_CHOSEN];
};
// The same by a workgroup, which needs a barrier for every count: four bounds at a time.  mine(b): how many keys of this wavefront are >= b; turn: of the two
// places for counts, so that one barrier is enough.
// Key is the value alone (32 bits, compared four times as fast) or all of a key.  False: more than `most` equal ones, of value `found`.
template <typename Key, int W, typename Mine>
__device__ __forceinline__ bool bound_of_all(Key lowest, Key above, int least, int most, Selection<W> &l, int &turn, Key &found, Mine &&mine) {
  Key lo = lowest, hi = above;
  for (bool first = true;; first = false) {
    const Key width = hi - lo;
    if (!first && width <= 1) { found = lo; return false; }
    Key bound[4];                          // an eighth of a binade below, one, eight, and all; then fifths
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const Key down = first ? (j < 3 ? (Key)1 << (8 * sizeof(Key) - 12 + 3 * j) : width) : width > 5 ? width / 5 * (j + 1) : (Key)(j + 1);
      bound[j] = down < width ? hi - down : first ? lo : lo + 1;
    }
    uint64_t packed = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) packed |= (uint64_t)mine(bound[j]) << (16 * j);
    if ((threadIdx.x & 63) == 0) l.counts[turn][threadIdx.x >> 6] = packed;
    __syncthreads();
    packed = 0;
#pragma unroll
    for (int k = 0; k < W; ++k) packed += l.counts[turn][k];
    turn ^= 1;
    if (first && (int)(packed >> 48) <= most) { found = lo; return true; }
    bool enough = false;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int n = (int)(packed >> (16 * j)) & 0xffff;
      if (enough) continue;
      if (n < least) { hi = bound[j]; continue; }
      if (n <= most) { found = bound[j]; return true; }
      enough = true;
      lo = bound[j];
    }
  }
}
template <int W, int N> __device__ __forceinline__ uint64_t bound_of_keys(const uint64_t (&key)[N], int used, uint64_t above, int top, Selection<W> &l, int &turn) {
  uint32_t value;
  const bool done = bound_of_all<uint32_t>(1, (uint32_t)(above >> 32) + 1, top, at_most(top), l, turn, value, [&](uint32_t bound) {
    int n = 0;
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (e < used) n += __popcll(__ballot((uint32_t)(key[e] >> 32) >= bound));
    return n;
  });
  if (done) return (uint64_t)value << 32;
  uint64_t found;
  bound_of_all<uint64_t>((uint64_t)value << 32, ((uint64_t)value << 32) + ((uint64_t)1 << 32), top, at_most(top), l, turn, found, [&](uint64_t bound) {
    int n = 0;
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (e < used) n += __popcll(__ballot(key[e] >= bound));
    return n;
  });
  return found;
}
// put(rank, key) for the first `top` of n keys in LDS, key 0 where there are fewer: four lanes count how many are larger than one of them
template <int THREADS, typename Put> __device__ __forceinline__ void put_in_order(const uint64_t *keys, int n, int top, int tid, Put &&put) {
  for (int i0 = 0; i0 < n; i0 += THREADS / 4) {
    const int i = i0 + (tid >> 2);
    const uint64_t key = keys[min(i, n - 1)];
    int rank = 0;
#pragma unroll 4
    for (int j = tid & 3; j < n; j += 4) rank += keys[j] > key ? 1 : 0;
    rank += __shfl_xor(rank, 1, 64);
    rank += __shfl_xor(rank, 2, 64);
    if (i < n && rank < top && (tid & 3) == 0) put(rank, key);
  }
  for (int i = n + tid; i < top; i += THREADS) put(i, (uint64_t)0);
}
// n candidates in LDS, in order
template <int W, typename Put> __device__ __forceinline__ void put_candidates(Selection<W> &l, int n, int top, uint64_t above, int &turn, Put &&put) {
  constexpr int THREADS = 64 * W, N = LP_CANDIDATES / THREADS;
  const int tid = threadIdx.x;
  if (n <= LP_CHOSEN) { put_in_order<THREADS>(l.candidate, n, top, tid, put); return; }
  uint64_t key[N];
#pragma unroll
  for (int e = 0; e < N; ++e) key[e] = e * THREADS + tid < n ? l.candidate[e * THREADS + tid] : 0;
  const uint64_t bound = bound_of_keys(key, (n + THREADS - 1) / THREADS, above, top, l, turn);
  if (tid == 0) l.n_chosen = 0;
  __syncthreads();
#pragma unroll
  for (int e = 0; e < N; ++e)
    if (key[e] >= bound) { const int k = atomicAdd(&l.n_chosen, 1); if (k < LP_CHOSEN) l.last[k] = key[e]; }
  __syncthreads();
  put_in_order<THREADS>(l.last, min(l.n_chosen, LP_CHOSEN), top, tid, put);
}

__device__ __forceinline__ void put_row(const LogProbsArgs &g, int64_t i, const RowStatistics &r) { g.stats[i] = r; g.entropy[i] = r.entropy; }
template <typename T> __device__ __forceinline__ void put_given(const LogProbsArgs &g, int64_t i, const RowStatistics &r, int j) {
  const int64_t tok = g.tokens[i * g.m + j];
  const T *z = static_cast<const T *>(g.z) + i * g.ld;
  g.log_probs[i * g.m + j] = tok >= 0 && tok < g.classes ? log_prob_of(load8(z, (int)tok, (int)tok + 1).v[0], r, g.tau) : 0.f;
}
// pad: the key's token is that much too large
__device__ __forceinline__ void put_top(const LogProbsArgs &g, int64_t i, const RowStatistics &r, int rank, uint64_t key, int pad = 0) {
  g.top_tokens[i * g.top + rank] = key ? key_token(key) - pad : -1;
  g.top_log_probs[i * g.top + rank] = log_prob_of(key ? key_logit(key) : -INFINITY, r, g.tau);
}
// of eight, NaN is passed over
__device__ __forceinline__ float largest_of(const f32x8 &x) {
  return fmaxf(fmaxf(fmaxf(x.v[0], x.v[1]), fmaxf(x.v[2], x.v[3])), fmaxf(fmaxf(x.v[4], x.v[5]), fmaxf(x.v[6], x.v[7])));
}
// Logits that lie before the first of a row up to a multiple of 16 bytes: a row is read from there on, in aligned pieces of eight, of which the first begins with `pad` masked
// ones.  (2048 x 50001 bf16 with pieces at odd addresses 49.3 us, so 43.5.)
template <typename T> __device__ __forceinline__ int row_pad(const T *z) { return (int)((reinterpret_cast<uintptr_t>(z) & 15) / sizeof(T)); }
// eight logits from o on, -infinity for what is not there
template <typename T> __device__ __forceinline__ f32x8 load_logits(const T *z, int o, int pad, int end) {
  f32x8 x;
  if (o >= pad && o + 8 <= end) return load8(z, o, 0x7fffffff);
#pragma unroll
  for (int e = 0; e < 8; ++e) x.v[e] = o + e >= pad && o + e < end ? load8(z, o + e, o + e + 1).v[0] : -INFINITY;
  return x;
}
// 2^x and x 2^x of eight logits from z = from
__device__ __forceinline__ void add_soft(const f32x8 &x, float from, float c, float &s, float &w) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float d = (x.v[e] - from) * c, p = __builtin_amdgcn_exp2f(d);
    s += p;
    w = fmaf(p, fmaxf(d, LP_NOTHING), w);
  }
}

// Up to 512 PIECES classes: a wavefront per row, which stays in registers, so that there is no barrier and a row is read once.  Bound by memory (32768 x 1000 float32 26.0 us, 5.05 TB/s),
// with most probable tokens by the LDS atomics and the orders of candidates (20 of 8192 x 999 bf16: 14.9 us, none 8.1; a workgroup per row 32.7).
template <typename T, int PIECES, bool TOP> __global__ __launch_bounds__(256) void log_probs_row_kernel(const LogProbsArgs g, int64_t rows) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t i = g.row0 + (int64_t)blockIdx.x * 4 + wave;
  if (i >= rows) return;
  const T *z = static_cast<const T *>(g.z) + i * g.ld;
  f32x8 x[PIECES];
  float largest[PIECES];
  SoftSums t = {-INFINITY, 0.f, 0.f};
#pragma unroll
  for (int p = 0; p < PIECES; ++p) {
    x[p] = load8(z, p * 512 + lane * 8, g.classes);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (p * 512 + lane * 8 + e >= g.classes) x[p].v[e] = -INFINITY;
    largest[p] = largest_of(x[p]);
    t.m = fmaxf(t.m, largest[p]);
  }
  t.m = wave_max(t.m);
#pragma unroll
  for (int p = 0; p < PIECES; ++p) add_soft(x[p], t.m == -INFINITY ? 0.f : t.m, g.c, t.s, t.w);
  t.s = wave_sum(t.s); t.w = wave_sum(t.w);
  const RowStatistics r = row_statistics(t);
  if (lane == 0) put_row(g, i, r);
  if (lane < g.m) put_given<T>(g, i, r, lane);

  if constexpr (TOP) {
    __shared__ uint64_t keys[4][LP_CHOSEN];
    __shared__ int4 table[4][LP_BINS / 4];
    uint64_t *const candidate = keys[wave];
    int *const bins = reinterpret_cast<int *>(table[wave]);
    // Pieces of eight first: as many as `top` of them within a bin hold the `top` largest, and an eighth of the atomics tells which bin.  Then the logits themselves.
    int n = LP_CHOSEN + 1;
    const auto choose = [&](auto &&add) {
      table[wave][lane] = table[wave][64 + lane] = make_int4(0, 0, 0, 0);
      wavefront_order();
      add();
      wavefront_order();
      const int by_bin = bin_bound(bins, g.top, lane);
      wavefront_order();
      if (by_bin == LP_BINS) return;
      n = 0;
#pragma unroll
      for (int e = 0; e < 8 * PIECES; ++e) {
        const float z = x[e >> 3].v[e & 7];
        const bool in = within_bin(z, t.m, g.c, by_bin);
        const uint64_t mask = __ballot(in);
        if (mask == 0) continue;
        const int to = n + lanes_before(mask);
        if (in && to < LP_CHOSEN) candidate[to] = logit_key(z, (e >> 3) * 512 + lane * 8 + (e & 7));
        n += __popcll(mask);
      }
    };
    const auto count_in = [&](float z) {
      const int bin = bin_of(z, t.m, g.c);
      if (bin < LP_BINS) atomicAdd(&bins[bin], 1);
    };
    choose([&]() {
#pragma unroll
      for (int p = 0; p < PIECES; ++p) count_in(largest[p]);
    });
    if (n > LP_CHOSEN) choose([&]() {
#pragma unroll
      for (int e = 0; e < 8 * PIECES; ++e) count_in(x[e >> 3].v[e & 7]);
    });
    if (n > LP_CHOSEN) {
      uint32_t order[8 * PIECES];
#pragma unroll
      for (int e = 0; e < 8 * PIECES; ++e) order[e] = (uint32_t)(logit_key(x[e >> 3].v[e & 7], 0) >> 32);
      const auto count = [&](uint32_t from) {
        int all = 0;
#pragma unroll
        for (int e = 0; e < 8 * PIECES; ++e) all += __popcll(__ballot(order[e] >= from));
        return all;
      };
      const int most = at_most(g.top);
      uint32_t bound = bound_of<uint32_t>(1, (uint32_t)(logit_key(t.m, 0) >> 32) + 1, 1u << 20, g.top, most, count);
      const bool ties = count(bound) > most;      // those above, and of equal ones the first
      if (ties) ++bound;
      const auto key = [&](int e) { return (uint64_t)order[e] << 32 | (0xffffffffu - (uint32_t)((e >> 3) * 512 + lane * 8 + (e & 7))); };
      n = 0;
#pragma unroll
      for (int e = 0; e < 8 * PIECES; ++e) {
        const bool in = order[e] >= bound;
        const uint64_t mask = __ballot(in);
        if (in) candidate[n + lanes_before(mask)] = key(e);
        n += __popcll(mask);
      }
      if (ties) {
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
          int mine = 0, before = 0;
#pragma unroll
          for (int e = 0; e < 8; ++e) mine += order[8 * p + e] == bound - 1 ? 1 : 0;
          int all = 0;
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            const uint64_t mask = __ballot((mine >> b) & 1);
            before += lanes_before(mask) << b; all += __popcll(mask) << b;
          }
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (order[8 * p + e] == bound - 1) {
              if (n + before < g.top) candidate[n + before] = key(8 * p + e);
              ++before;
            }
          n = min(n + all, g.top);
        }
      }
    }
    wavefront_order();
    put_in_order<64>(candidate, n, g.top, lane, [&](int rank, uint64_t k) { put_top(g, i, r, rank, k); });
  }
}

// A part of a row, one behind the other: `pieces` of eight logits for each thread, one of the workgroup's pieces behind the other.
constexpr int LP_STRIPS = 4, LP_MAX_PART = 131072, LP_MAX_PARTS = 64, LP_STEP = 2048;
constexpr float LP_SLACK = 8.f;            // x may be that far above its reference

// One workgroup per part.  One pass: sums about a reference that follows the largest at a distance, so that it hardly ever moves; and of every strip of pieces that a
// thread reads the largest logit and the first piece that has it.  The `top` largest strips hold the `top` most probable tokens (each has one of its own, and no token of
// another strip comes before any of them), so that the chosen strips alone are read again, and what reaches the bound is put in order.
// parts > 1: sums and keys of the part go to `sums` and `keys`, and log_probs_join_kernel ends the row.
// Bound by memory: 8192 x 131072 bf16 362 us (5.9 TB/s), with 20 tokens 376; ten vector operations and an exponential per logit take 0.28 ms of them.  (The first some 80 passes of a load
// that has just begun take up to 570.)  Four loads of a thread
// are on their way together.  Four strips a thread: with 20 tokens 7 % more is read; two cost as much, eight (fewer logits again, more of everything else) 396 and, for 8192 x 32000, 139
// instead of 114.  Few rows: 1 x 50000 with 20 tokens 9.9 us, of which the choice is 3.4 (table, strips again from L2, order).
struct LogPartArgs { LogProbsArgs g; int32_t parts, pieces; SoftSums *sums; uint64_t *keys; };

template <typename T, int W, bool TOP> __global__ __launch_bounds__(64 * W) void log_probs_kernel(const LogPartArgs a) {
  constexpr int AHEAD = 4, STEP = 512 * W;
  __shared__ float part_m[W], part_s[W], part_w[W];
  [[maybe_unused]] __shared__ Selection<W> l;
  const LogProbsArgs &g = a.g;
  const int64_t unit = g.row0 + blockIdx.x / (uint32_t)a.parts;
  const int part = (int)(blockIdx.x % (uint32_t)a.parts), tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const T *z = static_cast<const T *>(g.z) + unit * g.ld;
  const int pad = row_pad(z);
  z -= pad;
  const int begin = part * a.pieces * STEP, end = min(g.classes + pad, begin + a.pieces * STEP);
  const int per_strip = (a.pieces + LP_STRIPS - 1) / LP_STRIPS;

  float ref = -INFINITY, from = 0.f, s = 0.f, w = 0.f;         // from: ref, or 0 while there is none
  float largest[LP_STRIPS];
  int at[LP_STRIPS];
#pragma unroll
  for (int k = 0; k < LP_STRIPS; ++k) { largest[k] = -INFINITY; at[k] = 0; }
  const auto take = [&](const f32x8 &x, int piece, float &top, int &top_at) {
    const float m = largest_of(x);
    if (m > top) { top = m; top_at = piece; }
    if (__any((m - ref) * g.c > LP_SLACK)) {
      const float next = fmaxf(ref, m);
      if (ref != -INFINITY) { const SoftSums t = about({ref, s, w}, next, g.c); s = t.s; w = t.w; }
      ref = next;
      from = next == -INFINITY ? 0.f : next;
    }
    add_soft(x, from, g.c, s, w);
  };
#pragma unroll
  for (int k = 0; k < LP_STRIPS; ++k) {
    const int first = k * per_strip, last = min(a.pieces, first + per_strip);
    for (int q = first; q < last; q += AHEAD) {
      const int c = begin + q * STEP + tid * 8;
      if (begin + q * STEP >= end) break;
      if (q + AHEAD <= last && begin + (q + AHEAD) * STEP <= end && begin + q * STEP >= pad) {
        Raw8<T> raw[AHEAD];
#pragma unroll
        for (int e = 0; e < AHEAD; ++e) raw[e] = raw_load8(z, c + e * STEP, 0x7fffffff);
#pragma unroll
        for (int e = 0; e < AHEAD; ++e) take(expand8(raw[e]), q + e, largest[k], at[k]);
      } else {
        for (int e = 0; e < AHEAD && q + e < last; ++e) {
          const int o = c + e * STEP;
          if (o >= end) break;
          take(load_logits(z, o, pad, end), q + e, largest[k], at[k]);
        }
      }
    }
  }
  // From here on about the largest logit: about a reference 8 below it log p of a sure token would be the difference of two numbers of 8, three bits less exact.
  SoftSums t = {wave_max(fmaxf(fmaxf(largest[0], largest[1]), fmaxf(largest[2], largest[3]))), 0.f, 0.f};
  if constexpr (TOP) {
    for (int k = tid; k < LP_BINS; k += 64 * W) l.bins[k] = 0;
    if (tid == 0) l.n_chosen = l.n_candidates = 0;
  }
  if (lane == 0) part_m[wave] = t.m;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < W; ++k) t.m = fmaxf(t.m, part_m[k]);
  const float most = t.m;
  {
    const SoftSums u = about({ref, s, w}, most, g.c);
    t.s = wave_sum(u.s); t.w = wave_sum(u.w);
  }
  if (lane == 0) { part_s[wave] = t.s; part_w[wave] = t.w; }
  if constexpr (TOP) {
#pragma unroll
    for (int k = 0; k < LP_STRIPS; ++k) {
      const int bin = bin_of(largest[k], most, g.c);
      if (bin < LP_BINS) atomicAdd(&l.bins[bin], 1);
    }
  }
  __syncthreads();
  t.s = t.w = 0.f;
#pragma unroll
  for (int k = 0; k < W; ++k) { t.s += part_s[k]; t.w += part_w[k]; }
  const RowStatistics r = row_statistics(t);
  const int64_t out = unit * a.parts + part;
  if (a.parts == 1) {
    if (tid == 0) put_row(g, unit, r);
    if (tid < g.m) put_given<T>(g, unit, r, tid);
  } else if (tid == 0) a.sums[out] = t;

  if constexpr (TOP) {
    int turn = 0;
    const uint64_t above = logit_key(most, 0) + 1;
    const int by_bin = bin_bound(l.bins, g.top, lane);
    uint64_t bound = 1;
    bool chosen[LP_STRIPS];
    if (by_bin < LP_BINS) {
#pragma unroll
      for (int k = 0; k < LP_STRIPS; ++k) chosen[k] = within_bin(largest[k], most, g.c, by_bin);
    } else {
      uint64_t key[LP_STRIPS];
#pragma unroll
      for (int k = 0; k < LP_STRIPS; ++k) key[k] = logit_key(largest[k], begin + at[k] * STEP + tid * 8);
      bound = bound_of_keys(key, LP_STRIPS, above, g.top, l, turn);
#pragma unroll
      for (int k = 0; k < LP_STRIPS; ++k) chosen[k] = key[k] >= bound;
      // a strip's key is that of the first token of its piece: the others may come before the next strip's
      bound = max(bound & ~(uint64_t)7, (uint64_t)1);
    }
    // a wavefront's strips one behind the other
    uint64_t mask[LP_STRIPS];
    int mine = 0, place = 0;
#pragma unroll
    for (int k = 0; k < LP_STRIPS; ++k) { mask[k] = __ballot(chosen[k]); mine += __popcll(mask[k]); }
    if (lane == 0 && mine > 0) place = atomicAdd(&l.n_chosen, mine);
    place = __builtin_amdgcn_readfirstlane(place);
#pragma unroll
    for (int k = 0; k < LP_STRIPS; ++k) {
      const int n = place + lanes_before(mask[k]);
      if (chosen[k] && n < LP_CHOSEN) l.chosen[n] = k * 64 * W + tid;
      place += __popcll(mask[k]);
    }
    __syncthreads();
    const int strips = min(l.n_chosen, LP_CHOSEN), again = strips * per_strip;
    // eight logits of a chosen strip at a time
    const auto each = [&](auto &&f) {
      for (int i = tid; i < again; i += 64 * W) {
        const int u = i / strips, strip = l.chosen[i - u * strips], k = strip / (64 * W), q = k * per_strip + u, o = begin + q * STEP + (strip - k * 64 * W) * 8;
        if (q >= min(a.pieces, (k + 1) * per_strip) || o >= end) continue;
        const f32x8 x = load_logits(z, o, pad, end);
        uint64_t keys[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) keys[e] = by_bin == LP_BINS || within_bin(x.v[e], most, g.c, by_bin) ? logit_key(x.v[e], o + e) : 0;
        f(keys);
      }
    };
    const auto gather = [&](uint64_t b) {
      each([&](const uint64_t (&k)[8]) {
        int n = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) n += k[e] >= b ? 1 : 0;
        if (n == 0) return;
        int to = atomicAdd(&l.n_candidates, n);
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (k[e] >= b) { if (to < LP_CANDIDATES) l.candidate[to] = k[e]; ++to; }
      });
      __syncthreads();
    };
    gather(bound);
    if (l.n_candidates > LP_CANDIDATES) {  // many tokens of one strip: a bound among the tokens themselves
      const uint64_t from_strips = bound;
      bound_of_all<uint64_t>(from_strips, above, g.top, LP_CANDIDATES, l, turn, bound, [&](uint64_t b) {
        int n = 0;
        each([&](const uint64_t (&k)[8]) {
#pragma unroll
          for (int e = 0; e < 8; ++e) n += k[e] >= b ? 1 : 0;
        });
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) n += __shfl_xor(n, o, 64);
        return n;
      });
      __syncthreads();
      if (tid == 0) l.n_candidates = 0;
      __syncthreads();
      gather(bound);
    }
    put_candidates(l, min(l.n_candidates, LP_CANDIDATES), g.top, above, turn, [&](int rank, uint64_t k) {
      if (a.parts == 1) put_top(g, unit, r, rank, k, pad); else a.keys[out * g.top + rank] = k;
    });
  }
}

// The parts of a row together: sums in order, and of the keys those that reach a bound.
template <typename T> __global__ __launch_bounds__(256) void log_probs_join_kernel(const LogPartArgs a) {
  constexpr int N = LP_MAX_PARTS * LP_MAX_TOP / 256;
  __shared__ Selection<4> l;
  __shared__ float part_most[4];
  const LogProbsArgs &g = a.g;
  const int64_t i = g.row0 + blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63, n = a.parts * g.top, pad = row_pad(static_cast<const T *>(g.z) + i * g.ld);
  SoftSums t = {-INFINITY, 0.f, 0.f};
  if (lane < a.parts) t = a.sums[i * a.parts + lane];
  uint64_t key[N];
  float most = -INFINITY;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    key[e] = e * 256 + tid < n ? a.keys[i * n + e * 256 + tid] : 0;
    most = fmaxf(most, key[e] ? key_logit(key[e]) : -INFINITY);
  }
  t = about(t, wave_max(t.m), g.c);
  t.s = wave_sum(t.s); t.w = wave_sum(t.w);
  const RowStatistics r = row_statistics(t);
  if (tid == 0) put_row(g, i, r);
  if (tid < g.m) put_given<T>(g, i, r, tid);
  if (g.top == 0) return;
  most = wave_max(most);
  if (lane == 0) part_most[tid >> 6] = most;
  l.bins[tid] = l.bins[256 + tid] = 0;
  if (tid == 0) l.n_candidates = 0;
  __syncthreads();
  most = fmaxf(fmaxf(part_most[0], part_most[1]), fmaxf(part_most[2], part_most[3]));
  const int used = (n + 255) / 256;
  const auto bin = [&](uint64_t k) { return k ? bin_of(key_logit(k), most, g.c) : LP_BINS; };
#pragma unroll
  for (int e = 0; e < N; ++e)
    if (e < used && bin(key[e]) < LP_BINS) atomicAdd(&l.bins[bin(key[e])], 1);
  __syncthreads();
  int turn = 0;
  const uint64_t above = logit_key(most, 0) + 1;
  const int by_bin = bin_bound(l.bins, g.top, lane);
  const uint64_t bound = by_bin < LP_BINS ? 1 : bound_of_keys(key, used, above, g.top, l, turn);
#pragma unroll
  for (int e = 0; e < N; ++e)
    if (e < used && key[e] >= bound && (by_bin == LP_BINS || bin(key[e]) <= by_bin)) { const int k = atomicAdd(&l.n_candidates, 1); if (k < LP_CANDIDATES) l.candidate[k] = key[e]; }
  __syncthreads();
  put_candidates(l, min(l.n_candidates, LP_CANDIDATES), g.top, above, turn, [&](int rank, uint64_t k) { put_top(g, i, r, rank, k, pad); });
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
// W = 4: a workgroup per part of a row; W = 1: a wavefront per row, four rows a workgroup, for up to 4096 (bf16) or 3584 classes (32768 x 1000 bf16: 25 us, a workgroup per row 42).  A token's
// own part is added by the thread of its first appearance, with those of all others, behind the row's other values: no atomics, and the sum of a token that
// is given twice is rounded once.  Bound by memory: 4096 x 32000 bf16 106 us (5.0 TB/s, a copy's rate), 999 x 50001 float32 93 us; four loads of a thread
// together (two in a wavefront's row), 2 % better than two, and stores past the caches no better.
// LATE (1 / T above 2^64): 1 / T is a factor of the results and not of the coefficients: 0 times a coefficient over T that float32 does not hold would be no number.  (In one kernel for both:
// 999 x 50001 float32 1 % longer.)
template <typename T, int W, bool LATE> __global__ __launch_bounds__(256) void log_probs_grad_kernel(const LogProbsGradArgs g, int64_t rows) {
  constexpr int STEP = 512 * W, AHEAD = W == 1 ? 2 : 4;
  __shared__ int32_t tokens[4 / W][LP_MAX_TOKENS];
  __shared__ float coefs[4 / W][LP_MAX_TOKENS];
  const int which = W == 1 ? threadIdx.x >> 6 : 0, j = W == 1 ? threadIdx.x & 63 : threadIdx.x;
  const int64_t i = g.row0 + (W == 1 ? (int64_t)blockIdx.x * 4 + which : blockIdx.x / (uint32_t)g.parts);
  if (i >= rows) return;
  int32_t *const token = tokens[which];
  float *const a = coefs[which];
  const T *z = static_cast<const T *>(g.z) + i * g.ld;
  T *dz = static_cast<T *>(g.dz) + i * g.ld_dz;
  const int pad = row_pad(z);
  z -= pad; dz -= pad;
  const int begin = W == 1 ? 0 : (int)(blockIdx.x % (uint32_t)g.parts) * g.part_len, end = min(g.classes + pad, W == 1 ? 0x7fffffff : begin + g.part_len);
  if (begin >= end) return;
  const RowStatistics r = g.stats[i];
  const auto meet = [&]() { if constexpr (W == 1) { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup"); __builtin_amdgcn_wave_barrier(); } else __syncthreads(); };
  if (j < LP_MAX_TOKENS) {
    const int64_t t = j < g.m && g.a ? g.tokens[i * g.m + j] : -1;
    const bool valid = t >= 0 && t < g.classes;
    token[j] = valid ? (int32_t)t + pad : -1;
    a[j] = valid ? g.a[i * g.m + j] : 0.f;
  }
  meet();
  float all = 0.f, own = 0.f;
  bool first = j < LP_MAX_TOKENS && token[j] >= begin && token[j] < end;
  for (int k = 0; k < g.m; ++k) {
    all += a[k];
    if (first && token[k] == token[j]) { own += a[k]; if (k < j) first = false; }
  }
  const float before = LATE ? 1.f : g.tau, after = LATE ? g.tau : 1.f;
  const float b = g.b ? g.b[i] : 0.f, scale = -before * r.inv_s;
  const bool some = r.inv_s != 0.f && (all != 0.f || b != 0.f);
  const float k1 = some ? scale * b * LP_LN2 : 0.f, k0 = some ? scale * (all + b * (r.entropy - r.log2_s * LP_LN2)) : 0.f;
  const auto value = [&](float x) {
    const float d = fmaxf((x - r.m) * g.c, LP_NOTHING);
    return some ? __builtin_amdgcn_exp2f(d) * fmaf(k1, d, k0) : 0.f;
  };
  const auto put = [&](const Raw8<T> &raw, int v) {
    f32x8 x = expand8(raw);
#pragma unroll
    for (int e = 0; e < 8; ++e) x.v[e] = value(x.v[e]) * after;
    store8(dz, v, 0x7fffffff, x);
  };
  const auto one = [&](int v) { return value(load8(z, v, v + 1).v[0]); };
  const auto put_one = [&](int v, float y) { const f32x8 x = {{y}}; store8(dz, v, v + 1, x); };
  float at_token = 0.f;
  if (first) at_token = (one(token[j]) + (r.inv_s != 0.f ? before * own : 0.f)) * after;
  meet();
  int v = begin + j * 8;
  if (pad > 0 && v == 0) {                 // before the first whole piece
    for (int e = pad; e < min(8, end); ++e) put_one(e, one(e) * after);
    v += STEP;
  }
  for (; v + (AHEAD - 1) * STEP + 8 <= end; v += AHEAD * STEP) {
    Raw8<T> raw[AHEAD];
#pragma unroll
    for (int e = 0; e < AHEAD; ++e) raw[e] = raw_load8(z, v + e * STEP, 0x7fffffff);
#pragma unroll
    for (int e = 0; e < AHEAD; ++e) put(raw[e], v + e * STEP);
  }
  for (; v < end; v += STEP) {
    if (v + 8 <= end) put(raw_load8(z, v, 0x7fffffff), v);
    else for (int e = v; e < end; ++e) put_one(e, one(e) * after);
  }
  meet();
  if (first) put_one(token[j], at_token);
}

}  // namespace shampoo
