// libshampoo, the AdamW step and the norm of all gradients: argument checks, layout of the state, kernel launches and the extern "C" boundary of
// their part of shampoo.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <memory>
#include <new>
#include <type_traits>
#include <vector>

#include "adamw.h"
#include "host_checks.h"

using namespace shampoo;

struct shampoo_adamw {
  shampoo_adamw_config cfg;
  std::vector<int64_t> numel;
  std::vector<int64_t> first;        // chunk of a parameter, one more behind the last
  AdamState state;
  AdamChunk *chunks;
  int64_t last_step = -1;
};

namespace {

constexpr int64_t MAX_PARAMS = 1 << 20, MAX_ELEMENTS = (int64_t)1 << 39;      // the latter: 2 TiB of float32; pieces of 2^16 of them fit one launch
constexpr int64_t MAX_BLOCKS = 1 << 22;                                       // workgroups of a launch: its threads have 32 bits
constexpr int64_t NORM_CHUNK = 65536, NORM_LEAST = 2048;

// elements of all tensors; negative: an error code
int64_t total_of(int32_t n, const int64_t *numel) {
  int64_t total = 0;
  for (int32_t i = 0; i < n; ++i) {
    if (numel[i] < 0) return SHAMPOO_ERR_SHAPE;
    if (numel[i] > MAX_ELEMENTS || (total += numel[i]) > MAX_ELEMENTS) return SHAMPOO_ERR_UNSUPPORTED;
  }
  return total;
}
int check(const shampoo_adamw_config *c) {
  if (!c || !c->numel) return SHAMPOO_ERR_NULL;
  if (c->n_params < 1) return SHAMPOO_ERR_SHAPE;
  if (c->n_params > MAX_PARAMS) return SHAMPOO_ERR_UNSUPPORTED;
  const int64_t total = total_of(c->n_params, c->numel);
  if (total < 0) return (int)total;
  if (!dtype_ok(c->param_dtype) || !dtype_ok(c->grad_dtype) || (c->state_bits != 32 && c->state_bits != 8)) return SHAMPOO_ERR_HYPER;
  if (!(c->beta1 >= 0.0 && c->beta1 < 1.0 && c->beta2 >= 0.0 && c->beta2 < 1.0)) return SHAMPOO_ERR_HYPER;
  if (!(c->epsilon >= 1e-12 && c->epsilon <= 1e12 && c->weight_decay >= 0.0 && std::isfinite(c->weight_decay))) return SHAMPOO_ERR_HYPER;
  return SHAMPOO_OK;
}
int64_t groups_of(int64_t n) { return (n + AW_GROUP - 1) / AW_GROUP; }

size_t layout(const shampoo_adamw_config &c, void *workspace, AdamState &st, AdamChunk *&chunks, AdamTensor *&tensors) {
  int64_t total = 0, groups = 0, pieces = 0;
  for (int32_t i = 0; i < c.n_params; ++i) { total += c.numel[i]; groups += groups_of(c.numel[i]); pieces += (c.numel[i] + AW_CHUNK - 1) / AW_CHUNK; }
  Arena a(workspace);
  st = {};
  if (c.state_bits == 32) {
    st.m = a.take<float>((size_t)total);
    st.v = a.take<float>((size_t)total);
  } else {
    st.m8 = a.take<uint8_t>((size_t)(groups * AW_GROUP));
    st.v8 = a.take<uint8_t>((size_t)(groups * AW_GROUP));
    st.m_exp = a.take<uint8_t>((size_t)groups);
    st.v_exp = a.take<uint8_t>((size_t)groups);
  }
  chunks = a.take<AdamChunk>((size_t)pieces);
  tensors = a.take<AdamTensor>((size_t)c.n_params);
  return a.used;
}

// chunks c0 ... c1 - 1, at most MAX_BLOCKS in a launch
template <typename Launch> int by_chunks(int64_t c0, int64_t c1, Launch &&launch) {
  for (int64_t at = c0; at < c1; at += MAX_BLOCKS) {
    launch(at, dim3((unsigned)std::min(MAX_BLOCKS, c1 - at)));
    HIP_TRY(hipGetLastError());
  }
  return SHAMPOO_OK;
}
int set_states(shampoo_adamw *o, const float *m, const float *v, hipStream_t s) {
  return by_chunks(0, o->first.back(), [&](int64_t at, dim3 grid) {
    const AdamValuesArgs g = {o->chunks + at, o->state, const_cast<float *>(m), const_cast<float *>(v)};
    if (o->cfg.state_bits == 32) adamw_set_kernel<32><<<grid, 256, 0, s>>>(g); else adamw_set_kernel<8><<<grid, 256, 0, s>>>(g);
  });
}
template <typename P, typename G> void launch_step(int bits, dim3 grid, const AdamArgs &g, hipStream_t s) {
  if (bits == 32) adamw_kernel<P, G, 32><<<grid, 256, 0, s>>>(g); else adamw_kernel<P, G, 8><<<grid, 256, 0, s>>>(g);
}

// Elements of a piece of a sum of squares: eight pieces per CU where there is enough for that
int64_t norm_chunk(int64_t total) { return std::clamp<int64_t>(round_up(total / 2048, NORM_LEAST), NORM_LEAST, NORM_CHUNK); }
// pieces of all tensors; their number has 31 bits
int64_t norm_pieces(int32_t n, const int64_t *numel, int64_t chunk) {
  int64_t pieces = 0;
  for (int32_t i = 0; i < n; ++i) pieces += (numel[i] + chunk - 1) / chunk;
  return pieces;
}
int check_norm(int32_t n, const int64_t *numel, int64_t &chunk, int64_t &pieces) {
  if (n < 1) return SHAMPOO_ERR_SHAPE;
  if (!numel) return SHAMPOO_ERR_NULL;
  if (n > MAX_PARAMS) return SHAMPOO_ERR_UNSUPPORTED;
  const int64_t total = total_of(n, numel);
  if (total < 0) return (int)total;
  chunk = norm_chunk(total);
  pieces = norm_pieces(n, numel, chunk);
  return SHAMPOO_OK;
}
size_t norm_layout(int32_t n, int64_t pieces, void *workspace, double *&part, int32_t *&first) {
  Arena a(workspace);
  part = a.take<double>((size_t)pieces);
  first = a.take<int32_t>((size_t)n + 1);
  return a.used;
}

}  // namespace

extern "C" {

size_t shampoo_adamw_workspace_bytes(const shampoo_adamw_config *cfg) {
  if (check(cfg) != SHAMPOO_OK) return 0;
  AdamState st;
  AdamChunk *chunks;
  AdamTensor *tensors;
  return layout(*cfg, nullptr, st, chunks, tensors);
}

int shampoo_adamw_create(const shampoo_adamw_config *cfg, void *workspace, size_t workspace_bytes, void *stream, shampoo_adamw **out) try {
  if (!out) return SHAMPOO_ERR_NULL;
  *out = nullptr;
  TRY(check(cfg));
  std::unique_ptr<shampoo_adamw> o(new shampoo_adamw());
  o->cfg = *cfg;
  o->numel.assign(cfg->numel, cfg->numel + cfg->n_params);
  o->cfg.numel = o->numel.data();
  AdamTensor *table;
  TRY(workspace_ok(workspace, workspace_bytes, layout(o->cfg, workspace, o->state, o->chunks, table)));
  std::vector<AdamTensor> tensors;
  int64_t pieces = 0, flat = 0, slot = 0;
  for (int32_t i = 0; i < cfg->n_params; ++i) {
    const int64_t n = o->numel[i];
    o->first.push_back(pieces);
    tensors.push_back({pieces, n, flat, slot, !cfg->decay || cfg->decay[i] ? 1 : 0, 0});
    pieces += (n + AW_CHUNK - 1) / AW_CHUNK;
    flat += n;
    slot += groups_of(n) * AW_GROUP;
  }
  o->first.push_back(pieces);
  o->cfg.decay = nullptr;
  hipStream_t s = static_cast<hipStream_t>(stream);
  HIP_TRY(hipSetDevice(cfg->device));
  HIP_TRY(hipMemcpyAsync(table, tensors.data(), tensors.size() * sizeof(AdamTensor), hipMemcpyHostToDevice, s));
  if (pieces > 0) {
    adamw_chunks_kernel<<<dim3((unsigned)((pieces + 255) / 256)), 256, 0, s>>>(table, cfg->n_params, o->chunks, pieces);
    HIP_TRY(hipGetLastError());
  }
  TRY(set_states(o.get(), nullptr, nullptr, s));
  HIP_TRY(hipStreamSynchronize(s));
  *out = o.release();
  return SHAMPOO_OK;
} catch (...) {      // no host memory
  return SHAMPOO_ERR_HIP;
}

int shampoo_adamw_step(shampoo_adamw *o, void *const *params, const void *const *grads, void *const *copies, double lr, int64_t step, const float *norm,
                       float max_norm, void *stream) {
  if (!o || !params || !grads) return SHAMPOO_ERR_NULL;
  const shampoo_adamw_config &c = o->cfg;
  for (int32_t i = 0; i < c.n_params; ++i)
    if (c.numel[i] > 0 && (!params[i] || !grads[i] || (copies && !copies[i]))) return SHAMPOO_ERR_NULL;
  if (step < 0 || step <= o->last_step) return SHAMPOO_ERR_STEP;
  if (!std::isfinite(lr) || (norm && !(max_norm > 0.f))) return SHAMPOO_ERR_HYPER;
  if (copies && c.param_dtype != SHAMPOO_GRAD_F32) return SHAMPOO_ERR_HYPER;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const double t = (double)step + 1.0;
  AdamArgs g = {};
  g.state = o->state; g.norm = norm; g.max_norm = max_norm;
  g.b1 = (float)c.beta1; g.b1c = (float)(1.0 - c.beta1); g.b2 = (float)c.beta2; g.b2c = (float)(1.0 - c.beta2);
  g.inv_sqrt = (float)(1.0 / std::sqrt(1.0 - std::pow(c.beta2, t)));
  g.epsilon = (float)c.epsilon; g.keep = (float)(1.0 - lr * c.weight_decay); g.lr = (float)(lr / (1.0 - std::pow(c.beta1, t)));
  if (!std::isfinite(g.lr) || !std::isfinite(g.keep)) return SHAMPOO_ERR_HYPER;
  g.mix = (uint32_t)(uint64_t)step * AW_MIX2;
  g.has_copies = copies ? 1 : 0;
  const int32_t at_once = AW_POINTERS / (copies ? 3 : 2);
  for (int32_t i0 = 0; i0 < c.n_params; i0 += at_once) {
    const int32_t n = std::min(at_once, c.n_params - i0);
    g.tensor0 = i0; g.tensors = n;
    for (int32_t k = 0; k < n; ++k) {
      g.tensor[k] = params[i0 + k]; g.tensor[n + k] = grads[i0 + k];
      if (copies) g.tensor[2 * n + k] = copies[i0 + k];
    }
    TRY(by_chunks(o->first[i0], o->first[i0 + n], [&](int64_t at, dim3 grid) {
      g.chunks = o->chunks + at;
      const bool wide = c.grad_dtype == SHAMPOO_GRAD_F32;
      if (c.param_dtype == SHAMPOO_GRAD_F32) { if (wide) launch_step<float, float>(c.state_bits, grid, g, s); else launch_step<float, uint16_t>(c.state_bits, grid, g, s); }
      else { if (wide) launch_step<uint16_t, float>(c.state_bits, grid, g, s); else launch_step<uint16_t, uint16_t>(c.state_bits, grid, g, s); }
    }));
  }
  o->last_step = step;
  return SHAMPOO_OK;
}

int shampoo_adamw_get(shampoo_adamw *o, void *m, void *v, int32_t dtype, void *stream) {
  if (!o || (o->first.back() > 0 && (!m || !v))) return SHAMPOO_ERR_NULL;
  if (!dtype_ok(dtype)) return SHAMPOO_ERR_HYPER;
  hipStream_t s = static_cast<hipStream_t>(stream);
  return by_chunks(0, o->first.back(), [&](int64_t at, dim3 grid) {
    const AdamValuesArgs g = {o->chunks + at, o->state, m, v};
    if (dtype == SHAMPOO_GRAD_F32) { if (o->cfg.state_bits == 32) adamw_get_kernel<float, 32><<<grid, 256, 0, s>>>(g); else adamw_get_kernel<float, 8><<<grid, 256, 0, s>>>(g); }
    else { if (o->cfg.state_bits == 32) adamw_get_kernel<uint16_t, 32><<<grid, 256, 0, s>>>(g); else adamw_get_kernel<uint16_t, 8><<<grid, 256, 0, s>>>(g); }
  });
}

int shampoo_adamw_set(shampoo_adamw *o, const float *m, const float *v, void *stream) {
  if (!o || (o->first.back() > 0 && (!m || !v))) return SHAMPOO_ERR_NULL;
  return set_states(o, m, v, static_cast<hipStream_t>(stream));
}

int shampoo_adamw_destroy(shampoo_adamw *o) {
  if (!o) return SHAMPOO_ERR_NULL;
  delete o;
  return SHAMPOO_OK;
}

size_t shampoo_gradient_norm_workspace_bytes(int32_t n, const int64_t *numel) {
  int64_t chunk, pieces;
  if (check_norm(n, numel, chunk, pieces) != SHAMPOO_OK) return 0;
  double *part;
  int32_t *first;
  return norm_layout(n, pieces, nullptr, part, first);
}

int shampoo_gradient_norm(int32_t n, const void *const *grads, const int64_t *numel, int32_t dtype, float *norm, float *norms, void *workspace,
                          size_t workspace_bytes, void *stream) {
  if (!grads || !norm) return SHAMPOO_ERR_NULL;
  if (!dtype_ok(dtype)) return SHAMPOO_ERR_HYPER;
  int64_t chunk, pieces;
  TRY(check_norm(n, numel, chunk, pieces));
  for (int32_t i = 0; i < n; ++i)
    if (numel[i] > 0 && !grads[i]) return SHAMPOO_ERR_NULL;
  double *part;
  int32_t *first;
  TRY(workspace_ok(workspace, workspace_bytes, norm_layout(n, pieces, workspace, part, first)));
  hipStream_t s = static_cast<hipStream_t>(stream);
  int64_t block0 = 0;
  for (int32_t i0 = 0; i0 < n; i0 += GN_TENSORS) {
    NormArgs g = {};
    g.part = part; g.first = first; g.tensors = std::min(GN_TENSORS, n - i0); g.tensor0 = i0; g.block0 = (int32_t)block0; g.chunk = (int32_t)chunk;
    int64_t blocks = 0;
    for (int32_t k = 0; k < g.tensors; ++k) {
      g.at[k] = (int32_t)blocks; g.g[k] = grads[i0 + k]; g.len[k] = numel[i0 + k];
      blocks += (numel[i0 + k] + chunk - 1) / chunk;
    }
    g.blocks = (int32_t)blocks;
    const dim3 grid((unsigned)std::max<int64_t>(blocks, 1));
    if (dtype == SHAMPOO_GRAD_F32) square_sums_kernel<float><<<grid, 256, 0, s>>>(g); else square_sums_kernel<uint16_t><<<grid, 256, 0, s>>>(g);
    HIP_TRY(hipGetLastError());
    block0 += blocks;
  }
  norms_kernel<<<dim3((unsigned)n + 1), 1024, 0, s>>>(part, first, n, norm, norms);
  HIP_TRY(hipGetLastError());
  return SHAMPOO_OK;
}

}  // extern "C"
