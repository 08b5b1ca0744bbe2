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

int check(const shampoo_logits &c) {
  if (!dtype_ok(c.dtype) || !std::isfinite(c.inverse_temperature) || c.inverse_temperature <= 0.f) return SHAMPOO_ERR_HYPER;
  if (c.rows < 0 || c.classes < 1 || c.tokens < 0 || c.top < 0 || c.ld < c.classes) return SHAMPOO_ERR_SHAPE;
  if (c.rows > MAX_ROWS || c.classes > MAX_CLASSES || c.tokens > LP_MAX_TOKENS || c.top > LP_MAX_TOP) return SHAMPOO_ERR_UNSUPPORTED;
  return SHAMPOO_OK;
}
// 1 / T over log 2, of a T whose reciprocal float32 holds
float exponent_scale(float inverse_temperature) { return (float)((double)inverse_temperature * 1.4426950408889634); }

// rows at a time
template <typename Launch> int by_rows(int64_t rows, Launch &&launch) {
  for (int64_t r = 0; r < rows; r += MAX_BLOCKS) {
    launch(r, dim3((unsigned)std::min(MAX_BLOCKS, rows - r)));
    HIP_TRY(hipGetLastError());
  }
  return SHAMPOO_OK;
}

}  // namespace

extern "C" {

size_t shampoo_log_probs_workspace_bytes(const shampoo_logits *c) {
  return 0;
}

int shampoo_log_probs(const shampoo_logits *c, const void *logits, const int64_t *tokens, float *log_probs, float *entropy, int64_t *top_tokens,
                      float *top_log_probs, float *statistics, void *workspace, size_t workspace_bytes, void *stream) {
  if (!c) return SHAMPOO_ERR_NULL;
  TRY(check(*c));
  if (c->rows == 0) return SHAMPOO_OK;
  if (!logits || !entropy || !statistics || (c->tokens > 0 && (!tokens || !log_probs)) || (c->top > 0 && (!top_tokens || !top_log_probs))) return SHAMPOO_ERR_NULL;
  if (!aligned(statistics, 16)) return SHAMPOO_ERR_UNSUPPORTED;
  hipStream_t s = static_cast<hipStream_t>(stream);
  LogProbsArgs g = {};
  g.z = logits; g.ld = c->ld; g.tokens = tokens; g.c = exponent_scale(c->inverse_temperature); g.tau = c->inverse_temperature;
  g.classes = c->classes; g.m = c->tokens; g.top = c->top; g.log_probs = log_probs; g.entropy = entropy; g.top_tokens = top_tokens; g.top_log_probs = top_log_probs;
  g.stats = reinterpret_cast<RowStatistics *>(statistics);
  return by_rows(c->rows, [&](int64_t r, dim3 grid) {
    g.row0 = r;
    if (c->dtype == SHAMPOO_GRAD_F32) log_probs_kernel<float><<<grid, 256, 0, s>>>(g);
    else log_probs_kernel<uint16_t><<<grid, 256, 0, s>>>(g);
  });
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
  return by_rows(c->rows, [&](int64_t r, dim3 grid) {
    g.row0 = r;
    if (c->dtype == SHAMPOO_GRAD_F32) log_probs_grad_kernel<float><<<grid, 256, 0, s>>>(g);
    else log_probs_grad_kernel<uint16_t><<<grid, 256, 0, s>>>(g);
  });
}

}  // extern "C"
