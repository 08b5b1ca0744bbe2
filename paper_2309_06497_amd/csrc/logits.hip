// libshampoo, the operators on given logits: argument checks, workspace layout, kernel launches and the extern "C" boundary of their part of
// shampoo.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "host_checks.h"
#include "log_probs.h"

using namespace shampoo;

namespace {

constexpr int64_t MAX_ROWS = 0x7fffffff, MAX_BLOCKS = 1 << 22;      // workgroups of a launch: its threads have 32 bits
constexpr int32_t MAX_CLASSES = 1 << 22;

// 1 / T over log 2
float exponent_scale(float inverse_temperature) { return (float)((double)inverse_temperature * 1.4426950408889634); }
int check(const shampoo_logits &c) {
  if (!dtype_ok(c.dtype) || !(c.inverse_temperature > 0.f) || !std::isfinite(exponent_scale(c.inverse_temperature))) return SHAMPOO_ERR_HYPER;
  if (c.rows < 0 || c.classes < 1 || c.tokens < 0 || c.top < 0 || c.ld < c.classes) return SHAMPOO_ERR_SHAPE;
  if (c.rows > MAX_ROWS || c.classes > MAX_CLASSES || c.tokens > LP_MAX_TOKENS || c.top > LP_MAX_TOP) return SHAMPOO_ERR_UNSUPPORTED;
  return SHAMPOO_OK;
}

// The most logits before a row that its kernel skips to read aligned pieces
int32_t pad_of(const shampoo_logits &c, const void *logits) { return aligned(logits, 16) && c.ld * size_of(c.dtype) % 16 == 0 ? 0 : (int32_t)(16 / size_of(c.dtype)) - 1; }
// Parts of a row, in steps of `step` classes: what one workgroup takes at most, and where there are few rows as many as give four workgroups to every CU.
constexpr int64_t WORKGROUPS = 1024;
int32_t parts_of(int64_t rows, int32_t classes, int64_t step, int64_t longest, int64_t most_parts, int32_t pad, int32_t &pieces) {
  const int64_t all = (classes + pad + step - 1) / step;
  const int64_t wanted = std::max((classes + longest - 1) / longest, std::min(most_parts, (WORKGROUPS + rows - 1) / std::max<int64_t>(rows, 1)));
  pieces = (int32_t)((all + wanted - 1) / wanted);
  return (int32_t)((all + pieces - 1) / pieces);
}
// Rows of more classes than a wavefront keeps in registers have a workgroup each, of as many wavefronts as leave 16 pieces to a thread, or more where that fills the
// GPU's 4096 places.  20 tokens with 1, 2, 4 and 8 wavefronts: 8192 x 4096 bf16 28, 29, 38 and 59 us, 8192 x 131072 566, 466, 402 and 380, 1024 x 50000 51, 33, 29 and 26.
// Parts and a second launch for long rows where they are few.  Rows of 131072 bf16 classes in parts and whole, us: one 11.7 and 16.2 with 20 tokens, 8.1 and 12.3 with
// none; 63 rows 16.0 and 17.7, 9.0 and 14.1; 128 rows 19.2 and 18.1, 12.3 and 14.5; 256 rows 23.8 and 19.5, 16.3 and 15.7.  float32: one 11.5 and 15.3, 8.3 and 11.8; 63 rows
// 17.4 and 17.3, 10.5 and 13.8; 128 rows 21.7 and 18.6, 14.8 and 15.0.  50000 classes are faster whole in both types, for any number of rows: one 9.7 to 11.4.  So without
// alternatives parts would still pay at 128 rows, which this rule does not use.
constexpr int32_t SMALL_CLASSES = 2048, LONG_ROW = 65536;
constexpr int64_t FEW_ROWS = 64;
int wavefronts(int64_t rows, int32_t classes) {
  int w = 1;
  while (w < 8 && (classes > 8192 * w || (rows * w < 4096 && classes > 1024 * w))) w *= 2;
  return w;
}
size_t layout(const shampoo_logits &c, int32_t pad, void *workspace, LogPartArgs &a, int &w) {
  a.parts = 1;
  w = 0;
  if (c.classes <= SMALL_CLASSES) return 0;
  const bool cut = c.rows < FEW_ROWS && c.classes > LONG_ROW;
  w = cut ? 4 : wavefronts(c.rows, c.classes);
  a.parts = parts_of(c.rows, c.classes, 512 * w, LP_MAX_PART, cut ? LP_MAX_PARTS : 1, pad, a.pieces);
  Arena at(workspace);
  if (a.parts > 1) {
    a.sums = at.take<SoftSums>((size_t)(c.rows * a.parts));
    a.keys = at.take<uint64_t>((size_t)(c.rows * a.parts * c.top));
  }
  return at.used;
}

// rows at a time, `parts` workgroups each
template <typename Launch> int by_rows(int64_t rows, int32_t parts, Launch &&launch) {
  const int64_t at_once = MAX_BLOCKS / parts;
  for (int64_t r = 0; r < rows; r += at_once) {
    launch(r, (unsigned)std::min(at_once, rows - r));
    HIP_TRY(hipGetLastError());
  }
  return SHAMPOO_OK;
}
template <typename T, int W> void launch_parts(const LogPartArgs &a, unsigned n, hipStream_t s) {
  if (a.g.top > 0) log_probs_kernel<T, W, true><<<dim3(n * a.parts), 64 * W, 0, s>>>(a); else log_probs_kernel<T, W, false><<<dim3(n * a.parts), 64 * W, 0, s>>>(a);
}
template <typename T, int PIECES> void launch_rows(const LogProbsArgs &g, unsigned n, hipStream_t s) {
  const dim3 grid((n + 3) / 4);
  if (g.top > 0) log_probs_row_kernel<T, PIECES, true><<<grid, 256, 0, s>>>(g, g.row0 + n); else log_probs_row_kernel<T, PIECES, false><<<grid, 256, 0, s>>>(g, g.row0 + n);
}
template <typename T> int launch_log_probs(LogPartArgs a, int w, int64_t rows, hipStream_t s) {
  LogProbsArgs &g = a.g;
  TRY(by_rows(rows, a.parts, [&](int64_t r, unsigned n) {
    g.row0 = r;
    if (g.classes <= 512) launch_rows<T, 1>(g, n, s);
    else if (g.classes <= 1024) launch_rows<T, 2>(g, n, s);
    else if (g.classes <= SMALL_CLASSES) launch_rows<T, 4>(g, n, s);
    else switch (w) {
      case 1: launch_parts<T, 1>(a, n, s); break;
      case 2: launch_parts<T, 2>(a, n, s); break;
      case 4: launch_parts<T, 4>(a, n, s); break;
      default: launch_parts<T, 8>(a, n, s);
    }
  }));
  if (a.parts == 1) return SHAMPOO_OK;
  return by_rows(rows, 1, [&](int64_t r, unsigned n) {
    g.row0 = r;
    log_probs_join_kernel<T><<<dim3(n), 256, 0, s>>>(a);
  });
}
template <typename T, int W> void launch_grad_of(dim3 grid, const LogProbsGradArgs &g, int64_t rows, hipStream_t s) {
  if (g.tau > 0x1p64f) log_probs_grad_kernel<T, W, true><<<grid, 256, 0, s>>>(g, rows); else log_probs_grad_kernel<T, W, false><<<grid, 256, 0, s>>>(g, rows);
}
template <int W> void launch_grad(int32_t dtype, dim3 grid, const LogProbsGradArgs &g, int64_t rows, hipStream_t s) {
  if (dtype == SHAMPOO_GRAD_F32) launch_grad_of<float, W>(grid, g, rows, s); else launch_grad_of<uint16_t, W>(grid, g, rows, s);
}

}  // namespace

extern "C" {

size_t shampoo_log_probs_workspace_bytes(const shampoo_logits *c) {
  LogPartArgs a = {};
  int w;
  if (!c || check(*c) != SHAMPOO_OK) return 0;
  return std::max(layout(*c, 0, nullptr, a, w), layout(*c, 7, nullptr, a, w));      // whatever their alignment
}

int shampoo_log_probs(const shampoo_logits *c, const void *logits, const int64_t *tokens, float *log_probs, float *entropy, int64_t *top_tokens,
                      float *top_log_probs, float *statistics, void *workspace, size_t workspace_bytes, void *stream) {
  if (!c) return SHAMPOO_ERR_NULL;
  TRY(check(*c));
  if (c->rows == 0) return SHAMPOO_OK;
  if (!logits || !entropy || !statistics || (c->tokens > 0 && (!tokens || !log_probs)) || (c->top > 0 && (!top_tokens || !top_log_probs))) return SHAMPOO_ERR_NULL;
  if (!aligned(statistics, 16)) return SHAMPOO_ERR_UNSUPPORTED;
  LogPartArgs a = {};
  int w;
  TRY(workspace_ok(workspace, workspace_bytes, layout(*c, pad_of(*c, logits), workspace, a, w)));
  LogProbsArgs &g = a.g;
  g.z = logits; g.ld = c->ld; g.tokens = tokens; g.c = exponent_scale(c->inverse_temperature); g.tau = c->inverse_temperature;
  g.classes = c->classes; g.m = c->tokens; g.top = c->top; g.log_probs = log_probs; g.entropy = entropy; g.top_tokens = top_tokens; g.top_log_probs = top_log_probs;
  g.stats = reinterpret_cast<RowStatistics *>(statistics);
  hipStream_t s = static_cast<hipStream_t>(stream);
  return c->dtype == SHAMPOO_GRAD_F32 ? launch_log_probs<float>(a, w, c->rows, s) : launch_log_probs<uint16_t>(a, w, c->rows, s);
}

int shampoo_log_probs_grad(const shampoo_logits *c, const void *logits, const int64_t *tokens, const float *statistics, const float *d_log_probs,
                           const float *d_entropy, void *d_logits, int64_t ld_d_logits, void *stream) {
  if (!c) return SHAMPOO_ERR_NULL;
  TRY(check(*c));
  if (ld_d_logits < c->classes) return SHAMPOO_ERR_SHAPE;
  if (c->rows == 0) return SHAMPOO_OK;
  if (!logits || !statistics || !d_logits || (c->tokens > 0 && d_log_probs && !tokens)) return SHAMPOO_ERR_NULL;
  if (!aligned(statistics, 16)) return SHAMPOO_ERR_UNSUPPORTED;
  hipStream_t s = static_cast<hipStream_t>(stream);
  LogProbsGradArgs g = {};
  g.z = logits; g.ld = c->ld; g.tokens = tokens; g.stats = reinterpret_cast<const RowStatistics *>(statistics); g.a = d_log_probs; g.b = d_entropy;
  g.dz = d_logits; g.ld_dz = ld_d_logits; g.c = exponent_scale(c->inverse_temperature); g.tau = c->inverse_temperature;
  g.classes = c->classes; g.m = d_log_probs ? c->tokens : 0;
  int32_t pieces;
  // A wavefront per row: 32768 x 2100 bf16 52 us, a workgroup per row 96; 8192 x 4096 bf16 22.6, 23.4; 4096 x 4096 float32 26.8, 24.8; 4096 x 2100 float32 14.3, 16.4.
  if (c->classes <= (c->dtype == SHAMPOO_GRAD_F32 ? 3584 : 4096)) return by_rows(c->rows, 1, [&](int64_t r, unsigned n) {
    g.row0 = r;
    launch_grad<1>(c->dtype, dim3((n + 3) / 4), g, r + n, s);
  });
  g.parts = parts_of(c->rows, c->classes, LP_STEP, MAX_CLASSES, MAX_CLASSES, pad_of(*c, logits), pieces);
  g.part_len = pieces * LP_STEP;
  return by_rows(c->rows, g.parts, [&](int64_t r, unsigned n) {
    g.row0 = r;
    launch_grad<4>(c->dtype, dim3(n * g.parts), g, c->rows, s);
  });
}

}  // extern "C"
